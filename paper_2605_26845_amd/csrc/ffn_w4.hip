// moe_expert_ffn_w4_sliced: the experts' SwiGLU FFN over the row groups of a schedule with weights of 4 bits and one scale (and zero
// point) per group of 32, 64 or 128 inputs:   W[n][k] = (q[n][k] - zero[k / G][n]) * scale[k / G][n].
//
// A byte of two codes becomes a pair of bf16 values with a multiplication that copies it to the mantissas of both, a mask, and the exponent: without zero
// points (16 + q) units, the four bits above the lowest three of the mantissa; with zero points (48 + q - zero) units, where q and -zero are added above the lowest two, so
// that the exponent never changes.  Both exactly.  The matrix cores add products of these with x in fp32 over one group, starting at -24 (16 and the zero point 8)
// or -48 units times the group's sum of x, which one more product with a constant gives; and the scale multiplies that sum.  So no
// weight is ever rounded.  With a unit of 2^-12 every sum of a group stays finite for the largest finite x, whatever the signs: the codes' part is at most 31 * 128 units of it
// without zero points and 63 * 64 with them, the start 24 * 128 resp. 48 * 64, and the start with some of the products never more than the start.  Groups of 128 with
// zero points have twice these terms and a unit of 2^-13.
#include "lanes.hpp"
#include "plan.hpp"
#include "rows.hpp"
#include <algorithm>
#include <cmath>
#include <type_traits>

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int W4_STEP = 128;                    // values of K per step: 16 bytes of codes per lane, 16 weight rows
template <int G, bool ZERO> constexpr float CODE_UNITS = G == 128 && ZERO ? 0x1p13f : 0x1p12f;                      // in one
template <int G, bool ZERO> constexpr unsigned int START = G == 128 || !ZERO ? 0xBBC0BBC0u : 0xBC40BC40u;      // -24 or -48 units twice, in bf16: -24 * 2^-12 = -48 * 2^-13, or -48 * 2^-12

struct W4Args {
    const __bf16* x; __bf16* h; __bf16* y;      // h: [M][f] in schedule order
    const unsigned char *qg, *qu, *qd;
    const unsigned short *sg, *su, *sd;
    const unsigned char *zg, *zu, *zd;
    const int32_t* offsets;
    const int32_t* row_map; const float* row_gate;
    int M, S, E, d, f;
    // many rows: the plan's row blocks, or null (every workgroup finds its rows in the offsets; h lies in schedule order)
    const int4* blocks; int first_block, most_blocks;
    const int32_t* list; const float* list_gate;
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
    if (a.S == 1) {                                                       // its rows lie side by side
        int lo;
        total = group_rows(a.offsets, e, a.M, lo);
        for (int p = tid; p < min(total - first, ROWS); p += THREADS) s_row[p] = lo + first + p;
        moe::lds_only_barrier();
        return total;
    }
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
        moe::lds_only_barrier();                                           // (weights may be on their way)
        int base = total;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int t = s_scan[w];
            if (w < wave) base = add_rows(base, t, a.M);
            total = add_rows(total, t, a.M);
        }
        const int p0 = add_rows(base, incl, a.M) - rows;
        for (int p = max(p0, first); p < min(p0 + rows, first + ROWS); ++p) s_row[p - first] = lo + (p - p0);
        moe::lds_only_barrier();
    }
    return total;
}

// 16 bytes of codes per lane: lane (r16, g4) has k = 32 g4 .. 32 g4 + 31 of its weight row.  Afterwards a matrix instruction over dword i of all lanes stays
// inside a group: k8_of says which 8 values of K (of 128) lane group g4 holds in dword i.
template <int G> __device__ __forceinline__ void across_lanes(u32x4& c) {
    if constexpr (G <= 64) {
        const auto a = __builtin_amdgcn_permlane32_swap(c[0], c[2], false, false);
        const auto b = __builtin_amdgcn_permlane32_swap(c[1], c[3], false, false);
        c = u32x4{a[0], b[0], a[1], b[1]};
    }
    if constexpr (G == 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(c[0], c[1], false, false);
        const auto q = __builtin_amdgcn_permlane16_swap(c[2], c[3], false, false);
        c = u32x4{p[0], p[1], q[0], q[1]};
    }
}
template <int G> __device__ __forceinline__ int k8_of(int i, int g4) {
    if constexpr (G == 128) return 4 * g4 + i;
    if constexpr (G == 64) return (i >> 1) * 8 + 4 * (g4 & 1) + 2 * (g4 >> 1) + (i & 1);
    return 4 * i + g4;
}

// What code_values adds: without zero points the exponent of 16 units, else 48 units less the zero point
template <int G, bool ZERO> __device__ __forceinline__ unsigned int code_base(unsigned int zero) {
    return ZERO ? (G == 128 ? 0x3BC03BC0u : 0x3C403C40u) - (zero & 15u) * 0x00040004u : 0x3B803B80u;
}
// 8 codes (k, k + 1, .. from the lowest bits) -> 8 values; `mask` is MASK<ZERO> in a register of its own (an instruction holds one constant)
template <bool ZERO> constexpr unsigned int MASK = ZERO ? 0x003C003Cu : 0x00780078u;
template <bool ZERO> __device__ __forceinline__ bf16x8 code_values(unsigned int c, unsigned int base, unsigned int mask) {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const unsigned int both = ((c >> (8 * j)) & 0xFFu) * (ZERO ? 0x4004u : 0x8008u);
        if constexpr (ZERO) v[j] = __builtin_bit_cast(unsigned int, (u16x2)(__builtin_bit_cast(u16x2, both & mask) + __builtin_bit_cast(u16x2, base)));
        else v[j] = (both & mask) | base;
    }
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ bf16x8 splat(unsigned int two) { return __builtin_bit_cast(bf16x8, (u32x4{two, two, two, two})); }

// Of two neighbouring columns' scales and four columns' zero points as they lie in memory (whole words: a narrower load is extended, and waited for, before
// it is used), those of column `col`, as scale << 16 | zero
template <bool ZERO> __device__ __forceinline__ unsigned int scale_and_zero(unsigned int scales, unsigned int zeros, int col) {
    const unsigned int s = (col & 1) ? scales & 0xFFFF0000u : scales << 16;
    return ZERO ? s | ((zeros >> (8 * (col & 3))) & 0xFFu) : s;
}

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
// Bound by the weights' way from HBM.  A workgroup works through strips of 16 weight rows of one expert (phase 1: 8 gate and the 8 up rows of the same hidden
// units) for up to 16 of its rows; its W wavefronts share the contraction, 128 values of K each in turn, the codes straight from memory into the
// fragments of the matrix instruction, D - 1 steps ahead and across the strips.  The W partial sums of a strip meet in LDS and are added in a fixed
// order while the next strip's codes arrive.  x lies in LDS if it has room there (XLDS); otherwise its fragments are fetched a step ahead.
// One row of one expert, d 4096, f 14336, groups of 128 (88 MB of codes): phases 18 and 12 us, 3.3 and 2.4 TB/s, of which about 5 us each are the launch and the
// first trip to memory (the call takes tiles of 32 x 64 for the first, 17 us).  With zero points and groups of 32 or 64 up to 5 registers are spilled.  From registers alone, a strip per workgroup: 21 and 14; with a workgroup of 16 wavefronts 19 and 13.
template <int PHASE, int W, bool XLDS, int G, bool ZERO>
__global__ __attribute__((amdgpu_waves_per_eu(4))) __launch_bounds__(W * 64)
void ffn_w4_stream_kernel(W4Args a) {
    constexpr int NG = W4_STEP / G, PER = G / 32, D = 4;
    extern __shared__ __attribute__((aligned(16))) unsigned char s_x[];    // [min(M, 16)][K] bf16, rows 16 bytes further apart (banks)
    __shared__ int s_row[16];
    __shared__ int s_scan[W];
    __shared__ f32x4 s_red[2][W][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g4 = lane >> 4;
    const int e = blockIdx.y;
    const int K = PHASE == 1 ? a.d : a.f, NO = PHASE == 1 ? a.f : a.d;
    constexpr int COLS = PHASE == 1 ? 8 : 16;                              // output columns per strip
    const int strips = NO / COLS, mine = (strips - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
    const int KT = K / W4_STEP, n = (KT + W - 1) / W;                      // steps in all, and of a wavefront per strip (its last one may be none)
    const int steps = n * mine;
    unsigned int mask = MASK<ZERO>;
    asm("" : "+v"(mask));

    // lane r16's weight row: phase 1: gate rows in the lower half, up rows in the upper half of the 16
    const bool up = PHASE == 1 && r16 >= 8;
    const int row_in = PHASE == 1 ? r16 & 7 : r16;
    const unsigned char* const q = (PHASE == 2 ? a.qd : up ? a.qu : a.qg) + ((size_t)e * NO + row_in) * (size_t)(K / 2) + g4 * 16;
    const size_t group = (size_t)e * (K / G) * NO + (size_t)(g4 % NG) * NO;                // lane group g4 fetches group g4 % NG of the step
    const unsigned short* const sc = (PHASE == 2 ? a.sd : up ? a.su : a.sg) + group + (row_in & ~1);
    const unsigned char* const zp = ZERO ? (PHASE == 2 ? a.zd : up ? a.zu : a.zg) + group + (row_in & ~3) : nullptr;
    struct Codes { u32x4 q; unsigned int s, z; } codes[D];
    int next_strip = blockIdx.x, next_i = 0;                               // what is asked for next
    auto load_codes = [&](Codes& b) __attribute__((always_inline)) {
        // (a step that this wavefront does not have, or behind the last strip, asks for the step before it again: there is nothing new to fetch)
        const int kc = min(wave + W * next_i, KT - 1), strip = min(next_strip, strips - 1);
        b.q = *reinterpret_cast<const u32x4*>(q + (size_t)strip * COLS * (size_t)(K / 2) + kc * (W4_STEP / 2));
        const size_t so = (size_t)kc * NG * NO + strip * COLS;             // (strips are a multiple of 8 columns wide)
        b.s = *reinterpret_cast<const unsigned int*>(sc + so);
        if (ZERO) b.z = *reinterpret_cast<const unsigned int*>(zp + so);
        if (++next_i == n) { next_i = 0; next_strip += gridDim.x; }
    };
    // the first codes are asked for before the rows are known, where the expert can be expected to have any
    bool asked = a.E == 1 || a.M >= 4 * a.E;
    if (asked) {
#pragma unroll
        for (int u = 0; u < D - 1; ++u) load_codes(codes[u]);
    }
    for (int first = (int)blockIdx.z * 16;; first += (int)gridDim.z * 16) {
        const int rows = min(expert_rows<W * 64, 16>(a, e, first, s_row, s_scan) - first, 16);
        if (rows <= 0) return;
        if (!asked) {
            next_strip = blockIdx.x; next_i = 0;
#pragma unroll
            for (int u = 0; u < D - 1; ++u) load_codes(codes[u]);
        }
        asked = false;
        const __bf16* const xsrc = PHASE == 1 ? a.x : a.h;
        const int pitch = K * 2 + 16;
        if constexpr (XLDS) {                                              // (rows is at most M and 16, for which the host asks)
            const int per_row = K / 8, pieces = rows * per_row;
            for (int i0 = tid; i0 < pieces; i0 += W * 64 * 8) {            // 8 pieces of 16 bytes per thread on their way at once
                u32x4 v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int i = min(i0 + j * W * 64, pieces - 1), r = i / per_row, m = s_row[r];
                    v[j] = *reinterpret_cast<const u32x4*>(xsrc + (size_t)(PHASE == 1 ? w4_mapped(a, m) : m) * K + (i - r * per_row) * 8);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int i = i0 + j * W * 64, r = i / per_row;
                    if (i < pieces) *reinterpret_cast<u32x4*>(s_x + r * pitch + (i - r * per_row) * 16) = v[j];
                }
            }
            moe::lds_only_barrier();
        }
        const int my_row = s_row[min(r16, rows - 1)];                      // rows past the end repeat the last one and are not stored
        const __bf16* const xg = xsrc + (size_t)(PHASE == 1 ? w4_mapped(a, my_row) : my_row) * K;
        const unsigned char* const xl = s_x + min(r16, rows - 1) * pitch;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        u32x4 x[2][4];
        int x_i = 0;
        auto load_x = [&](u32x4 (&r)[4]) __attribute__((always_inline)) {
            const int kc = min(wave + W * x_i, KT - 1);
            if (++x_i == n) x_i = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = kc * W4_STEP + 8 * k8_of<G>(i, g4);
                if constexpr (XLDS) r[i] = *reinterpret_cast<const u32x4*>(xl + k * 2);
                else r[i] = *reinterpret_cast<const u32x4*>(xg + k);
            }
        };
        auto multiply = [&](Codes& b, const u32x4 (&r)[4]) __attribute__((always_inline)) {
            const bf16x8 constant = splat(START<G, ZERO>);
            f32x4 sum[NG];
#pragma unroll
            for (int i = 0; i < 4; ++i)                                    // what the group's sum starts at
                sum[i / PER] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r[i]), constant, i % PER == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sum[i / PER], 0, 0, 0);
            across_lanes<G>(b.q);
            unsigned int sz[NG];
            all_groups<NG>(scale_and_zero<ZERO>(b.s, b.z, row_in), sz);
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                const unsigned int base = code_base<G, ZERO>(sz[gr]);
#pragma unroll
                for (int i = gr * PER; i < (gr + 1) * PER; ++i)
                    sum[gr] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r[i]), code_values<ZERO>(b.q[i], base, mask), sum[gr], 0, 0, 0);
                const float scale = __builtin_bit_cast(float, sz[gr] & 0xFFFF0000u);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[v] = __builtin_fmaf(scale, sum[gr][v], acc[v]);
            }
        };
        // acc[v] of all wavefronts: row 4 * g4 + v, weight row r16 of the strip
        int half = 0, strip = blockIdx.x;
        auto finish = [&]() __attribute__((always_inline)) {
            s_red[half][wave][lane] = acc;
            acc = f32x4{0.f, 0.f, 0.f, 0.f};
            moe::lds_only_barrier();
            const float* const red = (const float*)s_red[half];
            if (tid < 16 * COLS) {
                const int col = tid % COLS, m16 = tid / COLS, at = ((m16 >> 2) * 16 + col) * 4 + (m16 & 3);
                if (m16 < rows) {
                    float s0 = red[at], s1 = 0.f;
#pragma unroll
                    for (int w = 1; w < W; ++w) s0 += red[w * 256 + at];
                    if (PHASE == 1) {
#pragma unroll
                        for (int w = 0; w < W; ++w) s1 += red[w * 256 + at + 32];
                    }
                    const int m = s_row[m16], o = strip * COLS + col;
                    // The hidden activation is rounded to bf16 once, as the operand of the second product, as in the library's other FFN calls: the results' error (2-norm, of their size)
                    // is 2.3e-3 with it and would be 1.7e-3 from y's own rounding; silu's reciprocal and exponential are the hardware's, a step each.
                    if (PHASE == 1) a.h[(size_t)m * a.f + o] = (__bf16)(silu(CODE_UNITS<G, ZERO> * s0) * (CODE_UNITS<G, ZERO> * s1));
                    else a.y[(size_t)w4_mapped(a, m) * a.d + o] = (__bf16)((a.row_gate ? a.row_gate[m] : 1.0f) * (CODE_UNITS<G, ZERO> * s0));
                }
            }
            half ^= 1;
            strip += gridDim.x;
        };
        load_x(x[0]);
        int i_now = 0;
        for (int j = 0; j < steps; j += D) {
#pragma unroll
            for (int u = 0; u < D; ++u) {
                if (j + u >= steps) break;
                load_x(x[(u + 1) & 1]);
                load_codes(codes[(u + D - 1) % D]);
                __builtin_amdgcn_sched_barrier(0);
                if (wave + W * i_now < KT) multiply(codes[u], x[u & 1]);
                __builtin_amdgcn_sched_barrier(0);
                if (++i_now == n) { i_now = 0; finish(); }
            }
        }
        __syncthreads();                                                   // s_row, s_x and s_red are used again
    }
}

// ---------------------------------------------------------------------------------- more rows per expert
// A workgroup takes up to 16 * TM rows of one expert and CW * NC * 16 weight rows; a wavefront NC tiles of 16 weight rows and all the rows, so
// that a code is widened once for up to 16 * TM rows.  The codes come straight from memory into registers, a step of K = 128 ahead.  x goes
// through LDS (two buffers; chunks of 16 bytes at place chunk ^ (row % 16) of a row, so that the 16 rows of a fragment lie in different
// banks).  KS slices of wavefronts share the contraction and add their sums in LDS at the end.
// Bound by issue: 4000 rows of d and f 4096, groups of 128, tiles of 64 x 256: 305 + 158 us (880 and 850 TFLOP/s), the matrix cores busy 52 % of the cycles (a fifth of it for the groups'
// sums of x), the vector instructions (widening 2 per pair of codes, with zero points 3, and a multiply-add per sum and group) 39 %, and little of both at once.  8191 rows of
// E 4, d 2048, f 1408: 114 and 71 us; groups of 32 with zero points, in tiles of 64 x 128, 188 and 104.  203 rows of E 4, d 7168, f 2048, groups of 32 with zero points, in tiles of
// 32 x 64: 54 and 37 us, vector instructions 56 % of the cycles; without loading x 47 + 29, without loading codes 48 + 30.
// Two workgroups per compute unit, not three, though smaller tiles leave registers for it: the dispatcher then loads some compute units with three and others with
// one (54 us above becomes 66).  Measured without a gain: codes or x further ahead; four slices; the sums of x through LDS, a step ahead (117 and 75 us at 8191 rows, 61 and 36 at 203); column
// tile by column tile, the codes of the next one widened between the products of this one (117 and 71); starting column tiles at different steps; h step by step in
// memory; a raised priority for the products; tiles of 128 x 128, which widen half as often (156 and 83 against 64 x 128's 150 and 83).  Tiles of 128 x 256 (one wavefront per SIMD, whose sums spill to the matrix cores' half of the registers and are copied for
// every multiply-add): 196 and 110.
template <int PHASE, int TM, int CW, int KS, int NC, int G, bool ZERO>
__global__ __attribute__((amdgpu_waves_per_eu(2, 2))) __launch_bounds__(CW * KS * 64)
void ffn_w4_tile_kernel(W4Args a) {
    static_assert(PHASE == 2 || NC % 2 == 0, "gate and up tiles in pairs");
    constexpr int THREADS = CW * KS * 64, TS = CW * 64, ROWS = 16 * TM, NI = ROWS * 16 / TS, NG = W4_STEP / G, PER = G / 32, D = 2, RB = NC == 4 ? 1 : 2;
    constexpr int NH = PHASE == 1 ? NC / 2 : NC;                           // column tiles of the output
    constexpr int X_BYTES = ROWS * 256, SLICE = 2 * X_BYTES;
    constexpr int RED_BYTES = (KS - 1) * CW * NC * TM * 64 * 16, LDS = KS * SLICE > RED_BYTES ? KS * SLICE : RED_BYTES;
    __shared__ __attribute__((aligned(16))) unsigned char s_mem[LDS];
    __shared__ int s_row[ROWS], s_io[ROWS];                                // row of h; of x (phase 1) and y (phase 2)
    __shared__ float s_gate[PHASE == 2 ? ROWS : 1];
    __shared__ int s_scan[THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g4 = lane >> 4, cw = wave % CW, ks = wave / CW;
    const int K = PHASE == 1 ? a.d : a.f, NO = PHASE == 1 ? a.f : a.d;
    unsigned int mask = MASK<ZERO>;
    asm("" : "+v"(mask));
    int e, rows, col_tile;
    for (int z = blockIdx.z;; z += gridDim.z) {                            // (a workgroup that follows a list has one block; so have the largest tiles, of whose registers a loop would spill more than the 4, with zero points 11, that are spilled)
        if (a.blocks) {
            // neighbouring workgroups of a die (every eighth one) take the column tiles of one row block, whose rows then stay in its L2; with few row blocks
            // the dies share them
            const int cols = NO / (CW * NH * 16), blocks = a.blocks[0].x, id = blockIdx.x;
            int block;
            if (blocks >= 32) { const int i = id >> 3; block = i / cols * 8 + (id & 7); col_tile = i % cols; }
            else { block = id / cols; col_tile = id % cols; }
            if (block >= blocks) return;
            const int4 b = a.blocks[a.first_block + block];
            e = __builtin_amdgcn_readfirstlane(b.z);
            rows = __builtin_amdgcn_readfirstlane(min(b.y - b.x, ROWS));
            for (int i = tid; i < rows; i += THREADS) {
                s_row[i] = b.x + i;
                s_io[i] = a.list[b.x + i];
                if (PHASE == 2) s_gate[i] = a.list_gate ? a.list_gate[b.x + i] : 1.0f;
            }
        } else {
            col_tile = blockIdx.x;
            e = blockIdx.y;
            const int first = z * ROWS;
            rows = min(expert_rows<THREADS, ROWS>(a, e, first, s_row, s_scan) - first, ROWS);
            if (rows <= 0) return;
            for (int i = tid; i < rows; i += THREADS) {
                const int m = s_row[i];
                s_io[i] = w4_mapped(a, m);
                if (PHASE == 2) s_gate[i] = a.row_gate ? a.row_gate[m] : 1.0f;
            }
        }
        __syncthreads();
        const int tiles = (rows + 15) / 16;
        const int col0 = (col_tile * CW + cw) * NH * 16;
        const int KT = K / W4_STEP, n = (KT - ks + KS - 1) / KS, n_most = (KT + KS - 1) / KS;      // steps of this slice, of any slice

        // ---- what a thread copies: chunk `chunk` of rows row0, row0 + TS / 16, ...
        const int ts = tid % TS, chunk = ts & 15, row0 = ts >> 4;
        const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)(PHASE == 1 ? (const void*)a.x : (const void*)a.h), 0, (unsigned int)a.M * (unsigned int)K * 2u, 0x00020000);
        unsigned int xoff[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int r = row0 + i * (TS / 16);
            xoff[i] = r < rows ? (unsigned int)(PHASE == 1 ? s_io[r] : s_row[r]) * (unsigned int)K * 2u + (unsigned int)chunk * 16u : 0xFFFFFF00u;      // past the end: zeros
        }
        const unsigned char* qbase[NC];
        const unsigned short* sbase[NC];
        const unsigned char* zbase[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = col0 + (c % NH) * 16;
            const size_t row = (size_t)e * NO + col, group = (size_t)e * (K / G) * NO + col;
            qbase[c] = (PHASE == 2 ? a.qd : c >= NH ? a.qu : a.qg) + row * (size_t)(K / 2);
            sbase[c] = (PHASE == 2 ? a.sd : c >= NH ? a.su : a.sg) + group;
            zbase[c] = ZERO ? (PHASE == 2 ? a.zd : c >= NH ? a.zu : a.zg) + group : nullptr;
        }
        const unsigned int qoff = (unsigned int)r16 * (unsigned int)(K / 2) + (unsigned int)g4 * 16u;
        const unsigned int soff = (unsigned int)(g4 % NG) * (unsigned int)NO + (unsigned int)r16;
        // The steps of this slice come round again behind its last one (what is loaded then is not used); a slice that has none (ks >= KT) starts at step 0.
        const int kstep = KS % KT;
        auto next_step = [&](int& kc) __attribute__((always_inline)) { kc += kstep; if (kc >= KT) kc -= KT; };
        int kx = n > 0 ? ks : 0, kq = kx;                                      // of the next x and of the next codes to be loaded

        struct Codes { u32x4 q[NC]; unsigned int s[NC], z[NC]; };
        auto load_codes = [&](Codes& b) __attribute__((always_inline)) {
            const unsigned int kc = (unsigned int)kq;
            next_step(kq);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const unsigned int so = soff + kc * NG * (unsigned int)NO;
                b.q[c] = *reinterpret_cast<const u32x4*>(qbase[c] + (qoff + kc * (W4_STEP / 2)));
                b.s[c] = *reinterpret_cast<const unsigned int*>(sbase[c] + (so & ~1u));
                if (ZERO) b.z[c] = *reinterpret_cast<const unsigned int*>(zbase[c] + (so & ~3u));
            }
        };
        auto work = [&](auto tag) __attribute__((always_inline)) {
            constexpr int T = decltype(tag)::value;                            // row tiles
            constexpr int TI = (T * 256 + TS - 1) / TS;                        // pieces of x a thread copies per step
            unsigned char* const mem = s_mem + ks * SLICE;
            u32x4 xr[TI];
            auto load_x = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < TI; ++j) xr[j] = __builtin_amdgcn_raw_buffer_load_b128(rx, xoff[j], kx * (W4_STEP * 2), 0);
                next_step(kx);
            };
            auto put_x = [&](int buffer) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < TI; ++j) {
                    const int row = row0 + j * (TS / 16);
                    *reinterpret_cast<u32x4*>(mem + buffer * X_BYTES + row * 256 + ((chunk ^ row) & 15) * 16) = xr[j];
                }
            };
            auto fragment = [&](int buffer, int t, int i) __attribute__((always_inline)) {
                const int row = t * 16 + r16;
                return *reinterpret_cast<const bf16x8*>(mem + buffer * X_BYTES + row * 256 + ((k8_of<G>(i, g4) ^ row) & 15) * 16);
            };
            const bf16x8 constant = splat(START<G, ZERO>);
            f32x4 acc[NC][T];
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int t = 0; t < T; ++t) acc[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
            auto multiply = [&](Codes& b, int buffer) __attribute__((always_inline)) {
                unsigned int sz[NC][NG];
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    across_lanes<G>(b.q[c]);
                    all_groups<NG>(scale_and_zero<ZERO>(b.s[c], b.z[c], r16), sz[c]);
                }
                // group by group, row tile by row tile, the fragments of the next row tile on their way from LDS (not more: registers)
                struct Rows { bf16x8 x[PER]; } rb[RB];
                auto fetch = [&](Rows& r, int gr, int t) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < PER; ++i) r.x[i] = fragment(buffer, t, gr * PER + i);
                };
                if (RB == 2) fetch(rb[0], 0, 0);
#pragma unroll
                for (int gr = 0; gr < NG; ++gr) {
                    bf16x8 w[NC][PER];
                    float scale[NC];
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        scale[c] = __builtin_bit_cast(float, sz[c][gr] & 0xFFFF0000u);
                        const unsigned int base = code_base<G, ZERO>(sz[c][gr]);
#pragma unroll
                        for (int i = 0; i < PER; ++i) w[c][i] = code_values<ZERO>(b.q[c][gr * PER + i], base, mask);
                    }
#pragma unroll
                    for (int t = 0; t < T; ++t) {
                        const int at = gr * T + t;
                        if (RB == 1) fetch(rb[0], gr, t);
                        else if (at + 1 < NG * T) fetch(rb[(at + 1) % RB], (at + 1) / T, (at + 1) % T);
                        const Rows& r = rb[at % RB];
                        f32x4 sum[NC], start = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int i = 0; i < PER; ++i) start = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r.x[i], constant, start, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < PER; ++i)
#pragma unroll
                            for (int c = 0; c < NC; ++c) sum[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r.x[i], w[c][i], i == 0 ? start : sum[c], 0, 0, 0);
#pragma unroll
                        for (int c = 0; c < NC; ++c)
#pragma unroll
                            for (int v = 0; v < 4; ++v) acc[c][t][v] = __builtin_fmaf(scale[c], sum[c][v], acc[c][t][v]);
                        if (PER * NC > 4) __builtin_amdgcn_sched_barrier(0);
                    }
                }
            };
            Codes codes[D];
            load_x();
#pragma unroll
            for (int i = 0; i < D - 1; ++i) load_codes(codes[i]);
            put_x(0);
            moe::lds_only_barrier();
            // step i: its x is in LDS; the buffer of step i + 1 was last read in step i - 1
            int buffer = 0;
            for (int i = 0; i < n_most; i += D) {
#pragma unroll
                for (int u = 0; u < D; ++u) {
                    if (i + u >= n_most) break;
                    load_x();
                    load_codes(codes[(u + D - 1) % D]);
                    __builtin_amdgcn_sched_barrier(0);
                    if (i + u < n) multiply(codes[u], buffer);
                    buffer ^= 1;
                    put_x(buffer);
                    moe::lds_only_barrier();
                }
            }
            if constexpr (KS > 1) {
                f32x4* const red = (f32x4*)s_mem;
                if (ks > 0) {
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int t = 0; t < T; ++t) red[((((ks - 1) * CW + cw) * NC + c) * T + t) * 64 + lane] = acc[c][t];
                }
                __syncthreads();
                if (ks > 0) return;
#pragma unroll
                for (int s = 1; s < KS; ++s)
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int t = 0; t < T; ++t) acc[c][t] += red[((((s - 1) * CW + cw) * NC + c) * T + t) * 64 + lane];
            }
            // ---- acc[c][t][v]: row 4 * g4 + v of row tile t, column r16 of column tile c
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int r = t * 16 + 4 * g4 + v;
                    if (r >= rows) continue;
#pragma unroll
                    for (int c = 0; c < NH; ++c) {
                        const int o = col0 + c * 16 + r16;
                        // (the hidden activation's rounding: see the streaming kernel)
                        if constexpr (PHASE == 1) a.h[(size_t)s_row[r] * a.f + o] = (__bf16)(silu(CODE_UNITS<G, ZERO> * acc[c][t][v]) * (CODE_UNITS<G, ZERO> * acc[NH + c][t][v]));
                        else a.y[(size_t)s_io[r] * a.d + o] = (__bf16)(s_gate[r] * (CODE_UNITS<G, ZERO> * acc[c][t][v]));
                    }
                }
        };
        // (row tiles beyond the last one are zeros, and not stored)
        if constexpr (TM == 4) {
            if (tiles <= 2) work(std::integral_constant<int, 2>{});
            else work(std::integral_constant<int, 4>{});
        } else {
            if (tiles <= 1) work(std::integral_constant<int, 1>{});
            else work(std::integral_constant<int, 2>{});
        }
        if (NC == 4 || a.blocks || rows < ROWS) return;                    // (a full block may be followed by another)
        __syncthreads();                                                   // s_row and the rest are used again
    }
}

// row blocks per expert that get a workgroup without a list: for three times the average (an expert with more keeps its workgroups for another block)
constexpr long long MOST_BLOCKS = 65535;          // of a grid's third dimension
int scanned_blocks(const W4Args& a, int rows) {
    const int held = std::max(1, std::min(a.E, a.M));
    return (int)std::min<long long>({(a.M - 1) / rows + 1, (3LL * a.M - 1) / ((long long)held * rows) + 1, MOST_BLOCKS});
}
template <int PHASE, int TM, int CW, int KS, int NC, int G, bool ZERO> moe_status launch_tile(const W4Args& a, hipStream_t s) {
    const int cols = (PHASE == 1 ? a.f : a.d) / (CW * 16 * (PHASE == 1 ? NC / 2 : NC));
    constexpr const char* NAMES[] = {"ffn_w4_small1_kernel", "ffn_w4_small2_kernel", "ffn_w4_middle1_kernel", "ffn_w4_middle2_kernel", "ffn_w4_large1_kernel", "ffn_w4_large2_kernel"};
    moe::LaunchScope k(NAMES[(TM == 2 ? 0 : NC == 2 ? 2 : 4) + PHASE - 1], s);
    // (the kernel deals rows to dies in groups of eight)
    const dim3 grid = a.blocks ? dim3((unsigned)cols * (unsigned)((a.most_blocks + 7) / 8 * 8)) : dim3(cols, a.E, NC == 4 ? (a.M - 1) / (16 * TM) + 1 : scanned_blocks(a, 16 * TM));
    hipLaunchKernelGGL((ffn_w4_tile_kernel<PHASE, TM, CW, KS, NC, G, ZERO>), grid, dim3(CW * KS * 64), 0, s, a);
    return k.done();
}

constexpr int STREAM_X_MOST = 124 * 1024;       // LDS for x, beside 16 KiB for the sums
constexpr int STREAM_W = 8;

// LDS for x in a streaming launch, 0 where it has no room
int stream_lds(const W4Args& a, int K) {
    const int lds = std::min(a.M, 16) * (K * 2 + 16);
    return lds <= STREAM_X_MOST ? lds : 0;
}
// two workgroups per compute unit, as far as their LDS allows, for the experts that can hold rows
dim3 stream_grid(const W4Args& a, int strips, int lds, int cus) {
    const int per_cu = lds > 60 * 1024 ? 1 : 2, held = std::max(1, std::min(a.E, a.M));
    return dim3(std::min(strips, std::max(1, cus * per_cu / held)), a.E, std::min((a.M - 1) / 16 + 1, 8));
}

template <int PHASE, bool XLDS, int G, bool ZERO> moe_status launch_stream(const W4Args& a, int lds, hipStream_t s) {
    auto kern = ffn_w4_stream_kernel<PHASE, STREAM_W, XLDS, G, ZERO>;
    if (XLDS) {
        static moe::DeviceOnce attr;
        int dev;
        if (attr.needed(dev)) {
            const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, STREAM_X_MOST);
            if (e != hipSuccess) { moe::note_hip_error(e, "hipFuncSetAttribute(MaxDynamicSharedMemorySize)"); return MOE_ERR_HIP; }
            attr.mark(dev);
        }
    }
    moe::LaunchScope k(PHASE == 1 ? "ffn_w4_stream1_kernel" : "ffn_w4_stream2_kernel", s);
    hipLaunchKernelGGL(kern, stream_grid(a, PHASE == 1 ? a.f / 8 : a.d / 16, lds, moe::compute_units()), dim3(STREAM_W * 64), lds, s, a);
    return k.done();
}

// ---- which kernel a phase takes, by estimates (us).  M bounds the rows; how they spread over the experts is not known here.
// Fitted to 168 shapes (E 1 .. 32, d 256 .. 7168, f 512 .. 14336, 1 .. 8191 rows, groups of 32, 64 and 128), every phase timed in every way; the choice takes 1.4 % longer than
// the best of them in the mean, and over 8 % longer in 8 shapes (one expert of 4096 x 4096 with 4 rows: 33 us against 26).  What a streaming workgroup costs that finds no rows was
// measured on 196 more (E 1 .. 2048, 1 .. 600 rows on experts of uneven popularity): 0.0031 us, so that one row on 128 experts of 2048 x 768 streams in 49 + 62 us and takes 13 + 15 in
// tiles of 32 x 64.  There the choice is 15 % behind in the mean and 2.4 times at most (one row on 2048 experts of 256 x 128: 31 against 13, of which the list 18; one on 128 of 7168 x 512: 56
// against 29; idle workgroups of the tiles cost half of what they are taken for with that many experts).  Streaming / tiles of 32 x 64 / 64 x 128 / 64 x 256, us, groups of
// 128, phase 1 + phase 2 (the tiles of 64 rows with a list of the rows, whose own launch takes 5 and with more rows up to 10):
//   E 1, d 4096, f 14336:   1 row 21+14  20+36  26+73  34+115,  12 rows 23+20  19+36  27+74  35+115,  96 rows 218+108  62+45  46+98  53+174,  400 rows -  227+107  150+101  132+175
//   E 4, d 7168, f 2048:    4 rows 21+14  21+11  38+14  57+18,  24 rows 35+18  24+12  40+15  58+19,   200 rows 143+55  41+29  55+25  89+29,   1000 rows -  148+104  111+51  120+43
//   E 4, d 2048, f 1408:    1 row 12+11  8+7  13+9  17+13,      200 rows 40+39  15+12  19+14  27+21,  2500 rows -  101+63  58+31  55+31,      8191 rows -  305+182  138+77  114+71
// (64 x 256 tiles in smaller groups: 2500 rows of the last, groups of 64, 67+36 and 81+40: the scales of more groups do not fit its registers.)
enum Way { W4_STREAM, W4_SMALL, W4_MIDDLE, W4_LARGE };
struct TileTimes { int rows, weight_rows, slices; double few, full, shared; };      // a step alone on its compute unit with up to half the rows, with all; its share of a full one
constexpr TileTimes SMALL_TILE = {32, 64, 2, 0.55, 0.82, 0.55}, MIDDLE_TILE = {64, 128, 1, 0.65, 0.90, 0.69}, LARGE_TILE = {64, 256, 1, 0.92, 1.53, 0.97};

struct Phase { int weight_rows, K; };
double tile_us(const TileTimes& c, const Phase& p, const W4Args& a, int group, bool planned, double cus) {
    const double held = std::max(1, std::min(a.E, a.M)), cols = p.weight_rows / c.weight_rows;
    const double blocks = std::max(held, a.M / (double)c.rows + 0.5 * held), steps = (p.K / W4_STEP + c.slices - 1) / c.slices;
    const double share = blocks * cols / cus, factor = group == 128 ? 1.0 : group == 64 ? 1.06 : 1.24;
    const double alone = a.M / held > c.rows / 2 ? c.full : c.few;
    double us = 3.3 + factor * steps * std::max(alone, c.shared * (share <= 2.0 ? std::ceil(share) : share));
    if (!planned) {
        us += std::max(0.0, a.E * (c.weight_rows == 256 ? std::ceil(a.M / (double)c.rows) : scanned_blocks(a, c.rows)) - blocks) * cols * 0.005;           // workgroups that find no rows
        us += 1.6 + a.S / 256 * 1.2 * std::max(1.0, share / 2);                                     // the walk over the slices
    }
    return us;
}
double stream_us(const Phase& p, const W4Args& a, int group, int cus) {
    const double held = std::max(1, std::min(a.E, a.M)), passes = std::ceil(std::min<double>(a.M, 3.0 * a.M / held) / 16);      // over the most popular expert's weights
    const double bytes = held * p.weight_rows * (p.K / 2.0) * (1.0 + 4.0 / group);
    const int lds = stream_lds(a, p.K);
    const dim3 grid = stream_grid(a, p.weight_rows / 16, lds, cus);
    const double idle = std::max(0.0, grid.x * ((double)grid.y * grid.z - held * std::min<double>(grid.z, passes)));      // workgroups that find no rows
    return 11.3 + passes * (bytes / 4.2e6) * (lds > 0 || a.M <= 4 ? 1.0 : 1.6) + a.S / 256 * 1.2 + idle * 0.0031;
}
// the best way of a phase, and its time
double best_way(const Phase& p, const W4Args& a, int group, bool planned, int cus, Way& way) {
    double least = 1e30;
    auto consider = [&](Way w, double us) { if (us < least) { least = us; way = w; } };
    if (!planned) {
        consider(W4_STREAM, stream_us(p, a, group, cus));
        consider(W4_SMALL, tile_us(SMALL_TILE, p, a, group, planned, cus));
    }
    consider(W4_MIDDLE, tile_us(MIDDLE_TILE, p, a, group, planned, cus));
    if (group == 128 && (planned || (a.M - 1) / LARGE_TILE.rows < MOST_BLOCKS)) consider(W4_LARGE, tile_us(LARGE_TILE, p, a, group, planned, cus));
    return least;
}

template <int PHASE, int G, bool ZERO> moe_status launch_way(Way way, const W4Args& a, hipStream_t s) {
    switch (way) {
        case W4_STREAM: {
            const int lds = stream_lds(a, PHASE == 1 ? a.d : a.f);
            return lds > 0 ? launch_stream<PHASE, true, G, ZERO>(a, lds, s) : launch_stream<PHASE, false, G, ZERO>(a, 0, s);
        }
        case W4_SMALL: return launch_tile<PHASE, 2, 2, 2, 2, G, ZERO>(a, s);
        case W4_LARGE:
            if constexpr (G == 128) return launch_tile<PHASE, 4, 4, 1, 4, G, ZERO>(a, s);
        default: return launch_tile<PHASE, 4, 4, 1, 2, G, ZERO>(a, s);
    }
}
template <int G, bool ZERO> moe_status both_phases(const W4Args& a, void* plan_at, hipStream_t s) {
    const Phase p1 = {2 * a.f, a.d}, p2 = {a.d, a.f};
    Way w1, w2, v1, v2;
    const int cus = moe::compute_units();
    const double scanned = best_way(p1, a, G, false, cus, w1) + best_way(p2, a, G, false, cus, w2);
    const double planned = best_way(p1, a, G, true, cus, v1) + best_way(p2, a, G, true, cus, v2) + 4.4 + a.M * 5e-4;
    W4Args p = a;
    if (planned < scanned) {                                               // a launch that lists the rows by expert, for both phases
        moe::RowsPlan plan = {a.offsets, a.S, a.E, a.M, 64, a.row_map, a.row_gate, nullptr, 0, nullptr, nullptr};
        if (const moe_status st = moe::rows_plan(plan, plan_at, s)) return st;
        p.blocks = plan.blocks; p.first_block = plan.first; p.most_blocks = a.M / 64 + a.E;
        p.list = plan.list; p.list_gate = plan.gate;
        w1 = v1; w2 = v2;
    }
    if (const moe_status st = launch_way<1, G, ZERO>(w1, p, s)) return st;
    return launch_way<2, G, ZERO>(w2, p, s);
}
template <int G> moe_status phases_of(const W4Args& a, void* plan_at, hipStream_t s) { return a.zg ? both_phases<G, true>(a, plan_at, s) : both_phases<G, false>(a, plan_at, s); }

size_t h_bytes(int M, int f) { return (((size_t)M * f * 2) + 255) & ~(size_t)255; }

constexpr int W4_MAX_GROUPS = 65536;

}  // namespace

extern "C" size_t moe_ffn_w4_workspace_bytes(int M, int d, int f) {
    if (M < 0 || d < 1 || f < 1) return 0;
    return h_bytes(M, f) + moe::rows_plan_bytes(M);
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
    if ((unsigned long long)M * std::max(d, f) * 2 >= 0xFFFFFF00ull) return MOE_ERR_UNSUPPORTED_SHAPE;      // rows are addressed with 32-bit offsets
    if (M == 0 || groups == 0) return MOE_OK;
    if (!x || !y) return MOE_ERR_INVALID_ARG;
    if ((((uintptr_t)x | (uintptr_t)y | (uintptr_t)q_gate | (uintptr_t)q_up | (uintptr_t)q_down | (uintptr_t)workspace) & 15) != 0) return MOE_ERR_INVALID_ARG;
    if ((((uintptr_t)s_gate | (uintptr_t)s_up | (uintptr_t)s_down | (uintptr_t)z_gate | (uintptr_t)z_up | (uintptr_t)z_down | (uintptr_t)row_map | (uintptr_t)row_gate |
          (uintptr_t)offsets) & 3) != 0) return MOE_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < moe_ffn_w4_workspace_bytes(M, d, f)) return MOE_ERR_WORKSPACE;
    const W4Args a = {(const __bf16*)x, (__bf16*)workspace, (__bf16*)y, (const unsigned char*)q_gate, (const unsigned char*)q_up, (const unsigned char*)q_down,
                      (const unsigned short*)s_gate, (const unsigned short*)s_up, (const unsigned short*)s_down, (const unsigned char*)z_gate,
                      (const unsigned char*)z_up, (const unsigned char*)z_down, offsets, row_map, row_gate, M, S, E_loc, d, f, nullptr, 0, 0, nullptr, nullptr};
    hipStream_t s = (hipStream_t)hip_stream;
    void* const plan_at = (char*)workspace + h_bytes(M, f);
    return group == 32 ? phases_of<32>(a, plan_at, s) : group == 64 ? phases_of<64>(a, plan_at, s) : phases_of<128>(a, plan_at, s);
}
