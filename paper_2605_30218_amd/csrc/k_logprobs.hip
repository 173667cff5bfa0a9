// k_logprobs.hip -- log probabilities of given tokens from rows of logits, with a row's entropy and its top alternatives.
//
// With m a row's largest logit, S = sum e^(x - m) and T = sum (x - m) e^(x - m):
//   log p(t) = x_t - m - ln S,  entropy = ln S - T / S,
// and the alternatives are the logits that come first by (value, then lower index).  One pass: a wave reads 2048 logits into
// registers, takes their sums under a running reference and moves those that beat the last of its `top` best into a list
// that it keeps sorted over its lanes; states and lists of a row's waves and segments join at the end.
#include <algorithm>

#include "mg_device.h"
#include "mg_kernels.h"

namespace mg {
namespace {

constexpr int LP_WAVES = 4;
constexpr int LP_THREADS = 64 * LP_WAVES;
constexpr int LP_PER = 32;              // logits of a lane
constexpr int LP_SUB = 64 * LP_PER;     // and of a wave at a time
constexpr int LP_MAX_SEGS = 64;
constexpr float LP_NONE = -__builtin_inff();

// (under-aligned vectors: rows begin anywhere)
struct __attribute__((packed, aligned(4))) LpF4 {
    float v[4];
};
struct __attribute__((packed, aligned(2))) LpH8 {
    uint16_t v[8];
};

// A candidate: value and index.  a before b: the larger value, the lower index among equal ones.
__device__ __forceinline__ bool lp_before(float av, int ai, float bv, int bi) { return av > bv || (av == bv && ai < bi); }

// The lists of a wave: lane i the i-th candidate.
struct LpList {
    float v;
    int i;
};
// the 64 first of two sorted lists, sorted; (rv, ri): the other list from its end
__device__ __forceinline__ void lp_merge(LpList& a, float rv, int ri) {
    const int lane = threadIdx.x & 63;
    if (lp_before(rv, ri, a.v, a.i)) {
        a.v = rv;
        a.i = ri;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const float v = __shfl_xor(a.v, o, 64);
        const int i = __shfl_xor(a.i, o, 64);
        const bool first = !(lane & o);  // this lane keeps the one that comes first
        if (lp_before(v, i, a.v, a.i) == first) {
            a.v = v;
            a.i = i;
        }
    }
}
// the k-th largest (from 0) of the lanes' values
__device__ __forceinline__ float lp_kth(float v, int k) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int n = 2; n <= 64; n <<= 1)
#pragma unroll
        for (int o = n >> 1; o >= 1; o >>= 1) {
            const float w = __shfl_xor(v, o, 64);
            const bool down = !(lane & n), low = !(lane & o);
            v = down == low ? fmaxf(v, w) : fminf(v, w);
        }
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), k));
}

// floats of a segment's state and list in the workspace
__host__ __device__ inline int lp_width(int top) { return 4 + (2 * top + 3) / 4 * 4; }

struct LpState {
    float m, S, T;
};
// S and T from reference `from` to `to`
__device__ __forceinline__ void lp_move(LpState& s, float to) {
    if (s.m > LP_NONE) {
        const float d = s.m - to, f = __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
        s.T = f == 0.0f ? 0.0f : f * (s.T + d * s.S);
        s.S = f * s.S;
    }
    s.m = to;
}

template <bool BF16>
struct LpRaw {
    uint32_t w[BF16 ? LP_PER / 2 : LP_PER];
};
// the index of value e of a lane, from the first of the wave's
template <bool BF16>
__device__ __forceinline__ int lp_index(int e, int lane) {
    return BF16 ? e / 8 * 512 + lane * 8 + e % 8 : e / 4 * 256 + lane * 4 + e % 4;
}
template <bool BF16>
__device__ __forceinline__ void lp_load(const void* row, int at, int end, int lane, LpRaw<BF16>& r) {
    if (BF16) {
        const uint16_t* p = static_cast<const uint16_t*>(row);
        if (at + LP_SUB <= end) {
#pragma unroll
            for (int j = 0; j < LP_PER / 8; ++j) {
                const LpH8 x = *reinterpret_cast<const LpH8*>(p + at + j * 512 + lane * 8);
#pragma unroll
                for (int i = 0; i < 4; ++i) r.w[4 * j + i] = x.v[2 * i] | (uint32_t)x.v[2 * i + 1] << 16;
            }
        } else {
#pragma unroll
            for (int i = 0; i < LP_PER / 2; ++i) {
                const int a = at + lp_index<true>(2 * i, lane);
                r.w[i] = (a < end ? p[a] : 0xff80u) | (a + 1 < end ? (uint32_t)p[a + 1] : 0xff80u) << 16;
            }
        }
    } else {
        const float* p = static_cast<const float*>(row);
        if (at + LP_SUB <= end) {
#pragma unroll
            for (int j = 0; j < LP_PER / 4; ++j) {
                const LpF4 x = *reinterpret_cast<const LpF4*>(p + at + j * 256 + lane * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) r.w[4 * j + i] = __float_as_uint(x.v[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < LP_PER; ++i) {
                const int a = at + lp_index<false>(i, lane);
                r.w[i] = a < end ? __float_as_uint(p[a]) : 0xff800000u;
            }
        }
    }
}
template <bool BF16>
__device__ __forceinline__ float lp_value(const LpRaw<BF16>& r, int e) {
    return BF16 ? (e & 1 ? bf_hi(r.w[e / 2]) : bf_lo(r.w[e / 2])) : __uint_as_float(r.w[e]);
}

// A row's results from its joined state and list.
template <bool BF16>
__device__ __forceinline__ void lp_finish(const LogpArgs& a, int64_t row, const LpState& s, const LpList& list) {
    const int lane = threadIdx.x & 63;
    const float ln = s.S == 0.0f ? 0.0f : logf(s.S);
    if (lane < a.top) {
        const bool some = list.v > LP_NONE;
        if (a.top_tokens) a.top_tokens[row * a.top + lane] = some ? list.i : -1;
        if (a.top_logprobs) a.top_logprobs[row * a.top + lane] = some ? (list.v - s.m) - ln : LP_NONE;
    }
    if (lane == 0) {
        if (a.entropy) a.entropy[row] = s.S == 0.0f ? 0.0f : ln - ieee_div(s.T, s.S);
        if (a.logprob) {
            const int t = a.tokens[row];
            float x = __builtin_nanf("");
            if (t >= 0 && t < a.V) {
                const int64_t at = row * a.stride + t;
                x = BF16 ? bf2f(static_cast<const uint16_t*>(a.logits)[at]) : static_cast<const float*>(a.logits)[at];
                // (a row that is masked whole has no reference)
                x = s.m == LP_NONE && s.S == 0.0f ? x : (x - s.m) - ln;
            }
            a.logprob[row] = x;
        }
    }
}

// One block a segment of a row; its waves take every LP_WAVES-th 2048 logits of it.  Alone in its row it writes the results, else
// its state and list.
template <bool BF16, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void logprobs_kernel(LogpArgs a, int segs) {
    __shared__ float sv[LP_WAVES][64], sm[LP_WAVES][3];
    __shared__ int si[LP_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x / segs;
    const int seg = blockIdx.x % segs;
    const int subs = (a.V + LP_SUB - 1) / LP_SUB;
    const int s0 = (int)((int64_t)subs * seg / segs), s1 = (int)((int64_t)subs * (seg + 1) / segs);
    const void* p = BF16 ? (const void*)(static_cast<const uint16_t*>(a.logits) + row * a.stride)
                         : (const void*)(static_cast<const float*>(a.logits) + row * a.stride);
    LpState st{LP_NONE, 0.0f, 0.0f};
    LpList list{LP_NONE, 0x7fffffff};
    float last = LP_NONE;  // the list's last value
    LpRaw<BF16> next;
    if (s0 + wave < s1) lp_load<BF16>(p, (s0 + wave) * LP_SUB, a.V, lane, next);
    for (int s = s0 + wave; s < s1; s += LP_WAVES) {
        const LpRaw<BF16> x = next;
        if (s + LP_WAVES < s1) lp_load<BF16>(p, (s + LP_WAVES) * LP_SUB, a.V, lane, next);
        float most = lp_value<BF16>(x, 0);
#pragma unroll
        for (int e = 1; e < LP_PER; ++e) most = fmaxf(most, lp_value<BF16>(x, e));
        const float top = fmaxf(st.m, wave_max(most));
        if (!(top <= LP_NONE)) {
            if (top != st.m) lp_move(st, top);
            float S = 0.0f, T = 0.0f;
#pragma unroll
            for (int e = 0; e < LP_PER; ++e) {
                const float y = lp_value<BF16>(x, e) - st.m, f = __builtin_amdgcn_exp2f(y * 1.4426950408889634f);
                S += f;
                T = __builtin_fmaf(f, fmaxf(y, -200.0f), T);  // (the factor of e^-inf is finite)
            }
            st.S += S;
            st.T += T;
        } else {  // nothing but -inf, or a NaN beside it
            float S = 0.0f;
#pragma unroll
            for (int e = 0; e < LP_PER; ++e) S += lp_value<BF16>(x, e) != lp_value<BF16>(x, e) ? 1.0f : 0.0f;
            if (__any(S != 0.0f)) st.S = __builtin_nanf("");
        }
        if (TOP) {
            float at = last;
            if (at == LP_NONE) at = lp_kth(most == most ? most : LP_NONE, a.top - 1);  // (at least `top` logits reach this one)
            if (__any(most >= at)) {
                const int base = s * LP_SUB;
#pragma unroll
                for (int e = 0; e < LP_PER; ++e) {
                    const float v = lp_value<BF16>(x, e);
                    unsigned long long hit = __ballot(v >= at && v > LP_NONE);
                    while (hit) {
                        const int l = __ffsll(hit) - 1;
                        hit &= hit - 1;
                        const float cv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l));
                        const int ci = base + lp_index<BF16>(e, l);
                        const int pos = __popcll(__ballot(lp_before(list.v, list.i, cv, ci)));
                        if (pos < a.top) {
                            const float uv = __shfl_up(list.v, 1, 64);
                            const int ui = __shfl_up(list.i, 1, 64);
                            list.v = lane < pos ? list.v : lane == pos ? cv : uv;
                            list.i = lane < pos ? list.i : lane == pos ? ci : ui;
                            last = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(list.v), a.top - 1));
                            at = fmaxf(at, last);
                        }
                    }
                }
            }
        }
    }
    // the waves join
    st.S = wave_sum_fast(st.S);
    st.T = wave_sum_fast(st.T);
    if (lane == 0) {
        sm[wave][0] = st.m;
        sm[wave][1] = st.S;
        sm[wave][2] = st.T;
    }
    if (TOP) {
        sv[wave][lane] = lane < a.top ? list.v : LP_NONE;
        si[wave][lane] = lane < a.top ? list.i : 0x7fffffff;
    }
    __syncthreads();
    if (wave) return;
    float m = sm[0][0];
#pragma unroll
    for (int w = 1; w < LP_WAVES; ++w) m = fmaxf(m, sm[w][0]);
    LpState sum{m, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < LP_WAVES; ++w) {
        LpState o{sm[w][0], sm[w][1], sm[w][2]};
        lp_move(o, m);
        sum.S += o.S;
        sum.T += o.T;
    }
    if (TOP) {
        list = LpList{sv[0][lane], si[0][lane]};
#pragma unroll
        for (int w = 1; w < LP_WAVES; ++w) lp_merge(list, sv[w][63 - lane], si[w][63 - lane]);
    }
    if (segs == 1) {
        lp_finish<BF16>(a, row, sum, list);
        return;
    }
    float* part = static_cast<float*>(a.part) + (int64_t)blockIdx.x * lp_width(a.top);
    if (lane == 0) *reinterpret_cast<float4*>(part) = make_float4(sum.m, sum.S, sum.T, 0.0f);
    if (TOP && lane < a.top) {
        part[4 + lane] = list.v;
        reinterpret_cast<int*>(part)[4 + a.top + lane] = list.i;
    }
}

// One block a row: its segments' states and lists join, a wave a list and then the waves pairwise.
constexpr int LP_JOIN_WAVES = 8;
template <bool BF16, bool TOP>
__global__ __launch_bounds__(64 * LP_JOIN_WAVES) void logprobs_join_kernel(LogpArgs a, int segs) {
    __shared__ float sv[LP_JOIN_WAVES][64];
    __shared__ int si[LP_JOIN_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x;
    const int width = lp_width(a.top);
    const float* part = static_cast<const float*>(a.part) + row * segs * width;
    LpList list{LP_NONE, 0x7fffffff};
    if (TOP) {
        for (int s = wave; s < segs; s += LP_JOIN_WAVES) {
            const float* q = part + (int64_t)s * width + 4;
            const int r = 63 - lane;
            const float rv = r < a.top ? q[r] : LP_NONE;
            const int ri = r < a.top ? reinterpret_cast<const int*>(q)[a.top + r] : 0x7fffffff;
            lp_merge(list, rv, ri);
        }
#pragma unroll
        for (int o = LP_JOIN_WAVES / 2; o >= 1; o >>= 1) {
            if (wave >= o && wave < 2 * o) {
                sv[wave][lane] = list.v;
                si[wave][lane] = list.i;
            }
            __syncthreads();
            if (wave < o) lp_merge(list, sv[wave + o][63 - lane], si[wave + o][63 - lane]);
        }
    }
    if (wave) return;
    LpState st{LP_NONE, 0.0f, 0.0f};
    if (lane < segs) {
        const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)lane * width);
        st = LpState{x.x, x.y, x.z};
    }
    lp_move(st, wave_max(st.m));
    st.S = wave_sum_fast(st.S);
    st.T = wave_sum_fast(st.T);
    lp_finish<BF16>(a, row, st, list);
}

// Segments of a row: until there are four blocks a CU, or every wave has one part.
int segments(const LogpArgs& a) {
    const int64_t subs = ((int64_t)a.V + LP_SUB - 1) / LP_SUB;
    const int64_t most = std::min<int64_t>((subs + LP_WAVES - 1) / LP_WAVES, LP_MAX_SEGS);
    return (int)std::max<int64_t>(1, std::min<int64_t>(most, (4 * a.n_cu + a.n - 1) / a.n));
}

template <bool BF16, bool TOP>
void launch(const LogpArgs& a, hipStream_t s) {
    const int segs = segments(a);
    hipLaunchKernelGGL((logprobs_kernel<BF16, TOP>), dim3((unsigned)((int64_t)a.n * segs)), dim3(LP_THREADS), 0, s, a, segs);
    if (segs > 1)
        hipLaunchKernelGGL((logprobs_join_kernel<BF16, TOP>), dim3((unsigned)a.n), dim3(TOP ? 64 * LP_JOIN_WAVES : 64), 0, s, a, segs);
}

}  // namespace

size_t logprobs_ws_bytes(const LogpArgs& a) {
    const int segs = segments(a);
    return segs == 1 ? 0 : (size_t)a.n * segs * lp_width(a.top) * sizeof(float);
}

hipError_t launch_logprobs(const LogpArgs& a, hipStream_t s) {
    auto f = a.bf16 ? (a.top ? launch<true, true> : launch<true, false>) : (a.top ? launch<false, true> : launch<false, false>);
    f(a, s);
    return hipGetLastError();
}

}  // namespace mg
