// moe_router_topk and its backward pass: the router of a MoE block (Section 2.1: each token is sent to its top-k experts), from logits to
// the expert ids that the histogram counts and the weights that the combine takes.
//
// LANES neighbouring lanes own a token and VPL neighbouring experts each: the logits are read once, 16 bytes at a time where a lane's neighbours are that many and rows start on 16
// bytes (4 float32 or 8 bf16 experts per lane and more), else one by one: with up to 16 experts, and in bf16 up to 64, and 129 to 256 for few tokens.  Every lane sorts
// its experts by (logit, lower index first); the largest head of all lanes is taken topk times, and the lane that held it moves its list up.
// (More than 4 experts per lane are looked through each time instead: sorting them is a quadratic number of exchanges.)
// Bound by the vector instructions of the choice, with few tokens by its chain: 32771 tokens of 64 experts, top-2, in bf16 6.8 us, 64 tokens of 256, top-8, 4.2 us.
// Neither the order of the lanes nor any atomic decides a tie: equal logits go to the lower index.
#include "lanes.hpp"
#include <algorithm>

namespace {

constexpr int ROUTER_THREADS = 256;

typedef __attribute__((ext_vector_type(4))) unsigned int r_u32x4;
typedef __attribute__((ext_vector_type(4))) float r_f32x4;

struct RouterArgs {
    const void* logits;
    const int32_t* ids_in;                     // backward
    const float* d_gates;                      // backward
    int32_t* ids;
    float* gates;
    void* d_logits;
    float scale;
    int T, E, topk, score, renormalise;
    int first;                                 // token of the first workgroup
};

// the first expert of this lane is e0; experts past the end and NaN count as masked
template <bool F32, int VPL, bool WIDE> __device__ __forceinline__ void read_logits(const void* p, size_t at, int e0, int E, float (&v)[VPL]) {
    constexpr int PIECE = F32 ? 4 : 8;                                     // values per 16 bytes
    if constexpr (WIDE && VPL % PIECE == 0) {
#pragma unroll
        for (int i = 0; i < VPL; i += PIECE) {
            if (e0 + i < E) {                                             // (E is a multiple of PIECE here)
                if constexpr (F32) {
                    const r_f32x4 r = *reinterpret_cast<const r_f32x4*>((const float*)p + at + i);
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[i + c] = r[c];
                } else {
                    const r_u32x4 r = *reinterpret_cast<const r_u32x4*>((const __bf16*)p + at + i);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        v[i + 2 * c] = __builtin_bit_cast(float, r[c] << 16);
                        v[i + 2 * c + 1] = __builtin_bit_cast(float, r[c] & 0xFFFF0000u);
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < PIECE; ++c) v[i + c] = -__builtin_inff();
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            v[i] = -__builtin_inff();
            if (e0 + i < E) v[i] = F32 ? ((const float*)p)[at + i] : (float)((const __bf16*)p)[at + i];
        }
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) v[i] = v[i] != v[i] ? -__builtin_inff() : v[i];
}

// a float as an unsigned number of the same order; 0 and -0 are the same, and the masked ones (-inf) become 0
__device__ __forceinline__ unsigned int order_key(float x) {
    const unsigned int u = __builtin_bit_cast(unsigned int, x + 0.0f);
    return x == -__builtin_inff() ? 0u : ((u & 0x80000000u) ? ~u : u | 0x80000000u);
}
__device__ __forceinline__ float key_value(unsigned int k) {
    return k == 0u ? -__builtin_inff() : __builtin_bit_cast(float, (k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }
// exp(x - top), top being at least x; equal infinities are as far apart as equal numbers
__device__ __forceinline__ float exp_below(float x, float top) { return x == top ? 1.0f : expf(x - top); }

// exp(x) for x <= 0 to 2 steps: x log2(e) in two parts, the hardware's power of two of the first, the second to first order (below 2^-126: zero)
__device__ __forceinline__ float exp_negative(float x) {
    const float y = fmaxf(x, -200.0f), t = y * 1.44269504f;
    const float r = __builtin_fmaf(y, 1.44269504f, -t) + y * 1.9259629e-8f, e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e, r * 0.693147182f, e);
}
__device__ __forceinline__ float exp_below_fast(float x, float top) { return x == top ? 1.0f : exp_negative(x - top); }

// sigmoid(x) / sigmoid(top) for x <= top, also where both are too small for a float
__device__ __forceinline__ float sigmoid_ratio(float x, float top) {
    const float ex = expf(-__builtin_fabsf(x)), et = expf(-__builtin_fabsf(top));
    return exp_below(fminf(x, 0.0f), fminf(top, 0.0f)) * (1.0f + et) / (1.0f + ex);
}

template <bool F32, int LANES, int VPL, bool WIDE>
__global__ __launch_bounds__(ROUTER_THREADS)
void router_topk_kernel(RouterArgs a) {
    const int sub = threadIdx.x % LANES;
    const long long t = a.first + (long long)blockIdx.x * (ROUTER_THREADS / LANES) + threadIdx.x / LANES;
    const bool live = t < a.T;                                             // (lanes of other tokens take part in the wavefront's exchanges)
    const int e0 = sub * VPL;
    float v[VPL];
    if (live) read_logits<F32, VPL, WIDE>(a.logits, (size_t)t * a.E + e0, e0, a.E, v);
    else {
#pragma unroll
        for (int i = 0; i < VPL; ++i) v[i] = -__builtin_inff();
    }
    // this lane's experts in falling order (a sort by exchanges of neighbours keeps equal ones in the order of their index)
    constexpr bool SORTED = VPL <= 4;
    unsigned int key[VPL], idx[SORTED ? VPL : 1], head, head_idx;
#pragma unroll
    for (int i = 0; i < VPL; ++i) key[i] = order_key(v[i]);
    auto look = [&]() __attribute__((always_inline)) {                     // the first of this lane's largest
        head = key[0]; head_idx = (unsigned)e0;
#pragma unroll
        for (int i = 1; i < VPL; ++i) {
            const bool more = key[i] > head;
            head = more ? key[i] : head;
            head_idx = more ? (unsigned)(e0 + i) : head_idx;
        }
    };
    if constexpr (SORTED) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) idx[i] = (unsigned)(e0 + i);
#pragma unroll
        for (int p = 0; p < VPL - 1; ++p)
#pragma unroll
            for (int i = VPL - 1; i > p; --i) {
                const bool up = key[i] > key[i - 1];
                const unsigned int k = key[i], x = idx[i];
                key[i] = up ? key[i - 1] : k; idx[i] = up ? idx[i - 1] : x;
                key[i - 1] = up ? k : key[i - 1]; idx[i - 1] = up ? x : idx[i - 1];
            }
        head = key[0]; head_idx = idx[0];
    } else {
        look();
    }
    const float top = key_value(moe::lanes_max<LANES>(head));
    float all = 0.0f;                                                      // sum of exp(logit - top) over all experts
    if (a.score == MOE_ROUTER_SOFTMAX && !a.renormalise) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) all += v[i] == -__builtin_inff() ? 0.0f : exp_below_fast(v[i], top);
        all = moe::lanes_sum<LANES>(all);
    }
    // lane j % LANES keeps slot j's choice
    constexpr int KEEP = (MOE_ROUTER_MAX_TOPK + LANES - 1) / LANES;
    unsigned int got_key[KEEP], got_idx[KEEP];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) got_key[i] = got_idx[i] = 0u;
    for (int j = 0; j < a.topk; ++j) {
        const unsigned int best = moe::lanes_max<LANES>(head);
        const unsigned int who = moe::lanes_min<LANES>(head == best ? head_idx : 0xFFFFFFFFu);
        if (sub == j % LANES) {
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
                if (i == j / LANES) { got_key[i] = best; got_idx[i] = who; }
        }
        const bool mine = head_idx == who;                                // (heads of zero are masked experts, whatever their index)
        if constexpr (SORTED) {
#pragma unroll
            for (int i = 0; i + 1 < VPL; ++i) { key[i] = mine ? key[i + 1] : key[i]; idx[i] = mine ? idx[i + 1] : idx[i]; }
            if (mine) { key[VPL - 1] = 0u; idx[VPL - 1] = 0xFFFFFFFEu; }
            head = key[0]; head_idx = idx[0];
        } else {
#pragma unroll
            for (int i = 0; i < VPL; ++i) key[i] = mine && who == (unsigned)(e0 + i) ? 0u : key[i];
            look();
        }
    }
    float w[KEEP], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const float x = key_value(got_key[i]);
        w[i] = 0.0f;
        if (got_key[i] != 0u) {
            if (a.score == MOE_ROUTER_SOFTMAX) w[i] = exp_below(x, top);
            else w[i] = a.renormalise ? sigmoid_ratio(x, top) : sigmoid(x);
        }
        sum += w[i];
    }
    if (a.renormalise) all = moe::lanes_sum<LANES>(sum);
    const float by = (a.renormalise || a.score == MOE_ROUTER_SOFTMAX) ? (all > 0.0f ? a.scale / all : 0.0f) : a.scale;
    if (live) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            const int j = i * LANES + sub;
            if (j < a.topk) {
                a.ids[(size_t)t * a.topk + j] = got_key[i] != 0u ? (int32_t)got_idx[i] : -1;
                a.gates[(size_t)t * a.topk + j] = w[i] * by;
            }
        }
    }
}

// LANES lanes per token (topk of them at least), which go through its experts in steps of LANES * VPL.  With G_j = scale d_gate_j over the slots whose expert is in range:
//   softmax                 d_l[e] = p_e (sum of G_j with id_j = e  -  sum_j G_j p_j)
//   renormalised (w_j sum to one over the slots)      d_l[id_j] += w_j (1 - sigmoid(l_j) for sigmoid scores, else 1) (G_j - sum_k G_k w_k)
//   sigmoid                 d_l[id_j] += G_j s_j (1 - s_j)
// What a slot gives its expert meets the expert's lane in LDS, a row of E floats per token.  Bound by the vector instructions of the exponentials: each is taken once
// (16384 tokens of 256 experts, top-8: 10.8 us, 3.1 TB/s; with a second one per logit, a wavefront per token and every lane asking every slot 16.5 us).
template <bool F32, int LANES, int VPL, bool WIDE>
__global__ __launch_bounds__(ROUTER_THREADS)
void router_backward_kernel(RouterArgs a) {
    extern __shared__ __attribute__((aligned(16))) float s_give[];
    const int sub = threadIdx.x % LANES;
    const long long t = a.first + (long long)blockIdx.x * (ROUTER_THREADS / LANES) + threadIdx.x / LANES;
    const bool live = t < a.T;                                             // (lanes of other tokens take part in the wavefront's exchanges)
    const size_t row = live ? (size_t)t * a.E : 0;
    const int pitch = (a.E + 3) & ~3;                                      // (16 bytes)
    float* const give_row = s_give + (threadIdx.x / LANES) * pitch;
    for (int e = sub * 4; e < a.E; e += LANES * 4) *reinterpret_cast<r_f32x4*>(give_row + e) = r_f32x4{0.f, 0.f, 0.f, 0.f};
    // lane j holds slot j
    int id = -1;
    float G = 0.0f, l = -__builtin_inff();
    if (live && sub < a.topk) {
        id = a.ids_in[(size_t)t * a.topk + sub];
        if ((unsigned)id < (unsigned)a.E) {
            G = a.scale * a.d_gates[(size_t)t * a.topk + sub];
            l = F32 ? ((const float*)a.logits)[row + id] : (float)((const __bf16*)a.logits)[row + id];
        }
        if (!(l > -__builtin_inff())) { id = -1; G = 0.0f; l = -__builtin_inff(); }      // a masked expert has a weight of zero whatever its logit
    }
    const bool dense = a.score == MOE_ROUTER_SOFTMAX && !a.renormalise;
    float top = -__builtin_inff(), all = 0.0f;
    float first[VPL], first_top = -__builtin_inff();                      // this lane's exponentials of the first step, over its own largest
#pragma unroll
    for (int i = 0; i < VPL; ++i) first[i] = 0.0f;
    if (dense && live) {
        // maximum and sum of the softmax in one pass over the row, then over the lanes
        for (int e = sub * VPL; e < a.E; e += LANES * VPL) {
            float v[VPL];
            read_logits<F32, VPL, WIDE>(a.logits, row + e, e, a.E, v);
            float m = top;
#pragma unroll
            for (int i = 0; i < VPL; ++i) m = fmaxf(m, v[i]);
            if (m != -__builtin_inff()) {
                all *= top == -__builtin_inff() ? 0.0f : exp_below_fast(top, m);
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    v[i] = v[i] == -__builtin_inff() ? 0.0f : exp_below_fast(v[i], m);
                    all += v[i];
                }
                top = m;
            } else {
#pragma unroll
                for (int i = 0; i < VPL; ++i) v[i] = 0.0f;
            }
            if (e < LANES * VPL) {
                first_top = top;
#pragma unroll
                for (int i = 0; i < VPL; ++i) first[i] = v[i];
            }
        }
    }
    const float mine = dense ? top : l;
    const float most = key_value(moe::lanes_max<LANES>(order_key(mine)));
    if (dense) all = moe::lanes_sum<LANES>(top == -__builtin_inff() ? 0.0f : all * exp_below_fast(top, most));
    top = most;
    float w = 0.0f, slope = 1.0f;
    if (id >= 0) {
        if (a.score == MOE_ROUTER_SOFTMAX) w = exp_below_fast(l, top);
        else {
            w = a.renormalise ? sigmoid_ratio(l, top) : sigmoid(l);
            slope = sigmoid(-l);
        }
    }
    if (a.renormalise) all = moe::lanes_sum<LANES>(w);
    if (a.renormalise || dense) w = all > 0.0f ? w / all : 0.0f;
    const float mean = moe::lanes_sum<LANES>(G * w);
    // what slot j's expert gets beside the dense part
    const float give = dense ? G : w * slope * (a.renormalise ? G - mean : G);
    // Each slot puts its number at its expert's place; who finds another one there shares the expert, and then the slots add theirs one after the other.
    // (One wavefront's LDS accesses are in order; the compiler must not know better.)
    asm volatile("" ::: "memory");
    if (id >= 0) give_row[id] = __builtin_bit_cast(float, 0x7F800001 + sub);
    asm volatile("" ::: "memory");
    const bool shared = id >= 0 && __builtin_bit_cast(int, give_row[id]) != 0x7F800001 + sub;
    asm volatile("" ::: "memory");
    if (__ballot(shared) == 0ull) {
        if (id >= 0) give_row[id] = give;
    } else {
        if (id >= 0) give_row[id] = 0.0f;
        for (int j = 0; j < a.topk; ++j) {
            asm volatile("" ::: "memory");
            if (id >= 0 && sub == j) give_row[id] += give;
        }
    }
    asm volatile("" ::: "memory");
    const float by = all > 0.0f ? exp_below_fast(first_top, top) / all : 0.0f;
    if (!live) return;
    for (int e = sub * VPL; e < a.E; e += LANES * VPL) {
        float o[VPL];
#pragma unroll
        for (int i = 0; i < VPL; ++i) o[i] = e + i < a.E ? give_row[e + i] : 0.0f;
        if (dense) {
            if (e < LANES * VPL) {
#pragma unroll
                for (int i = 0; i < VPL; ++i) o[i] = first[i] * by * (o[i] - mean);
            } else {
                float v[VPL];
                read_logits<F32, VPL, WIDE>(a.logits, row + e, e, a.E, v);
#pragma unroll
                for (int i = 0; i < VPL; ++i) o[i] = v[i] == -__builtin_inff() ? 0.0f : exp_below_fast(v[i], top) / all * (o[i] - mean);
            }
        }
        constexpr int PIECE = F32 ? 4 : 8;
        if constexpr (WIDE && VPL % PIECE == 0) {
#pragma unroll
            for (int i = 0; i < VPL; i += PIECE) {
                if (e + i >= a.E) continue;
                if constexpr (F32) {
                    *reinterpret_cast<r_f32x4*>((float*)a.d_logits + row + e + i) = r_f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]};
                } else {
                    typedef __attribute__((ext_vector_type(8))) __bf16 r_bf16x8;
                    r_bf16x8 b;
#pragma unroll
                    for (int c = 0; c < 8; ++c) b[c] = (__bf16)o[i + c];
                    *reinterpret_cast<r_u32x4*>((__bf16*)a.d_logits + row + e + i) = __builtin_bit_cast(r_u32x4, b);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (e + i < a.E) {
                    if constexpr (F32) ((float*)a.d_logits)[row + e + i] = o[i];
                    else ((__bf16*)a.d_logits)[row + e + i] = (__bf16)o[i];
                }
        }
    }
}

constexpr int MOST_TOKENS = 1 << 24;              // per launch, whose threads are counted in 32 bits
template <bool F32, int LANES, int VPL> moe_status launch_topk(RouterArgs a, bool wide, hipStream_t s) {
    constexpr int PER = ROUTER_THREADS / LANES;
    moe::LaunchScope k("router_topk_kernel", s);
    for (long long first = 0; first < a.T; first += MOST_TOKENS) {
        a.first = (int)first;
        const dim3 grid((unsigned)((std::min<long long>(a.T - first, MOST_TOKENS) - 1) / PER + 1)), block(ROUTER_THREADS);
        if (wide) hipLaunchKernelGGL((router_topk_kernel<F32, LANES, VPL, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((router_topk_kernel<F32, LANES, VPL, false>), grid, block, 0, s, a);
    }
    return k.done();
}
template <bool F32> moe_status topk_of(const RouterArgs& a, bool wide, hipStream_t s) {
    // (Times with the events around the launch, about 0.6 us more than the kernel's.)  16 experts per lane cost the fewest instructions (32768 tokens of 128 experts, top-6: 8 lanes 12.6 us, 16 lanes of 8 experts 20; 16384 of 256, top-8: 16 lanes 14.4, 32 of 8
    // 26, 64 of 4 21; 8192 of 512: 32 lanes 14, 64 of 8 25), four sorted ones per lane the shortest chain (64 tokens of 256: 4.8 against 7.1, level at some 4000 tokens).
    // Up to 64 experts the two are near each other and the chain counts: 32768 tokens of 64, top-2, 16 lanes of 4 7.4 us, 8 of 8 8.5, 4 of 16 7.8, top-8 8.9, 8.5 and 9.0; 4096 tokens, top-8,
    // 6.9, 8.3 and 7.9
    if (a.E <= 16) return launch_topk<F32, 16, 1>(a, wide, s);
    if (a.E <= 64) return launch_topk<F32, 16, 4>(a, wide, s);
    if (a.E <= 128) return launch_topk<F32, 8, 16>(a, wide, s);
    if (a.E <= 256) return a.T < 4096 ? launch_topk<F32, 64, 4>(a, wide, s) : launch_topk<F32, 16, 16>(a, wide, s);
    if (a.E <= 512) return launch_topk<F32, 32, 16>(a, wide, s);
    if (a.E <= 1024) return launch_topk<F32, 64, 16>(a, wide, s);
    return launch_topk<F32, 64, 64>(a, wide, s);
}

template <bool F32, int LANES, int VPL> moe_status launch_backward(RouterArgs a, bool wide, hipStream_t s) {
    constexpr int PER = ROUTER_THREADS / LANES;
    moe::LaunchScope k("router_backward_kernel", s);
    const int lds = PER * ((a.E + 3) & ~3) * (int)sizeof(float);           // (64 KiB for the most experts)
    for (long long first = 0; first < a.T; first += MOST_TOKENS) {
        a.first = (int)first;
        const dim3 grid((unsigned)((std::min<long long>(a.T - first, MOST_TOKENS) - 1) / PER + 1)), block(ROUTER_THREADS);
        if (wide) hipLaunchKernelGGL((router_backward_kernel<F32, LANES, VPL, true>), grid, block, lds, s, a);
        else hipLaunchKernelGGL((router_backward_kernel<F32, LANES, VPL, false>), grid, block, lds, s, a);
    }
    return k.done();
}
template <bool F32> moe_status backward_of(const RouterArgs& a, bool wide, hipStream_t s) {
    // as few lanes per token as its experts and slots leave (32768 tokens of 64 experts: 16 lanes 7.4 us, 64 lanes 16.1; 16384 of 256: 32 lanes of 8 experts 10.5, 64 of 4
    // 11.1, 16 of 16 13.6)
    if (a.topk <= 16 && a.E <= 64) return launch_backward<F32, 16, 4>(a, wide, s);
    if (a.topk <= 16 && a.E <= 128) return launch_backward<F32, 16, 8>(a, wide, s);
    if (a.E <= 256) return launch_backward<F32, 32, 8>(a, wide, s);
    return launch_backward<F32, 64, 8>(a, wide, s);
}

moe_status checked(int T, int E, int topk, int logits_type, int score, int flags, float scale) {
    if (T < 0 || E < 1 || topk < 1 || topk > E) return MOE_ERR_INVALID_ARG;
    if (logits_type != MOE_T_BF16 && logits_type != MOE_T_F32) return MOE_ERR_INVALID_ARG;
    if ((score != MOE_ROUTER_SOFTMAX && score != MOE_ROUTER_SIGMOID) || (flags & ~MOE_ROUTER_RENORMALISE) || !(__builtin_fabsf(scale) < __builtin_inff())) return MOE_ERR_INVALID_ARG;
    if (E > MOE_MAX_EXPERTS || topk > MOE_ROUTER_MAX_TOPK) return MOE_ERR_UNSUPPORTED_SHAPE;
    return MOE_OK;
}

}  // namespace

extern "C" moe_status moe_router_topk(const void* logits, int logits_type, int T, int E, int topk, int score, int flags, float scale, int32_t* ids, float* gates, void* hip_stream) {
    if (const moe_status st = checked(T, E, topk, logits_type, score, flags, scale)) return st;
    if (T == 0) return MOE_OK;
    const bool f32 = logits_type == MOE_T_F32;
    if (!logits || !ids || !gates || ((uintptr_t)logits & (f32 ? 3 : 1)) != 0 || (((uintptr_t)ids | (uintptr_t)gates) & 3) != 0) return MOE_ERR_INVALID_ARG;
    const RouterArgs a = {logits, nullptr, nullptr, ids, gates, nullptr, scale, T, E, topk, score, flags & MOE_ROUTER_RENORMALISE, 0};
    // rows start on 16 bytes: pieces of 16 bytes, else one value at a time
    const bool wide = ((uintptr_t)logits & 15) == 0 && E % (f32 ? 4 : 8) == 0;
    return f32 ? topk_of<true>(a, wide, (hipStream_t)hip_stream) : topk_of<false>(a, wide, (hipStream_t)hip_stream);
}

extern "C" moe_status moe_router_topk_backward(const float* d_gates, const void* logits, int logits_type, const int32_t* ids, int T, int E, int topk, int score, int flags,
                                               float scale, void* d_logits, void* hip_stream) {
    if (const moe_status st = checked(T, E, topk, logits_type, score, flags, scale)) return st;
    if (T == 0) return MOE_OK;
    const bool f32 = logits_type == MOE_T_F32;
    if (!d_gates || !logits || !ids || !d_logits || ((((uintptr_t)logits | (uintptr_t)d_logits) & (f32 ? 3 : 1)) != 0) || (((uintptr_t)ids | (uintptr_t)d_gates) & 3) != 0) return MOE_ERR_INVALID_ARG;
    const RouterArgs a = {logits, ids, d_gates, nullptr, nullptr, d_logits, scale, T, E, topk, score, flags & MOE_ROUTER_RENORMALISE, 0};
    const bool wide = (((uintptr_t)logits | (uintptr_t)d_logits) & 15) == 0 && E % (f32 ? 4 : 8) == 0;
    hipStream_t s = (hipStream_t)hip_stream;
    return f32 ? backward_of<true>(a, wide, s) : backward_of<false>(a, wide, s);
}
