// k_logprobs.hip -- log probabilities of given tokens from rows of logits, with a row's entropy and its top alternatives.
//
// With m a row's largest logit, S = sum e^(x - m) and T = sum (x - m) e^(x - m):
//   log p(t) = x_t - m - ln S,  entropy = ln S - T / S,
// and the alternatives are the logits that come first by (value, then lower index).  One pass: a wave reads 2048 logits into
// registers, takes their sums under a running reference and moves those that beat the last of its `top` best into a list
// that it keeps sorted over its lanes; states and lists of a row's waves and segments join at the end.  A list that starts empty
// would take in some hundred logits one after the other before its last keeps most out, so the waves of a block first agree on a
// value that `top` of their logits reach: the least of what enough lanes' largest reach in each wave.
//
// What bounds it: the logits' bytes where rows are many (2001 rows of 152064 bf16 with 8 alternatives 128 us, 4.75 TB/s, 2001 of
// 32000 fp32 with 20 49.7 us, 5.2 TB/s; a large read reaches 6.1), and where they are few the chain of load, floor, list, join and the second
// launch (one row of 128256 fp32 with 5 alternatives 9.7 us, the join alone 3; 64 rows with 20 16.1 us, 9.2 without alternatives).
// Exponentials take the logits' differences from the reference in 32 bits; nothing is rounded to fewer.
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
// A row is cut into segments until so many blocks a CU are there: 64 rows of 128256 fp32 logits with 20 alternatives take 16.0 us with 4 and
// 17.1 with 2, 256 such rows 34.2 and 34.1, one row 9.7 either way.
constexpr int LP_BLOCKS_PER_CU = 4;
constexpr float LP_NONE = -__builtin_inff();

// (under-aligned vectors: rows begin anywhere)
struct __attribute__((packed, aligned(4))) LpF4 {
    float v[4];
};
struct __attribute__((packed, aligned(2))) LpH8 {
    uint16_t v[8];
};

// The value of the lane whose number differs in bit O, and of the lane before (0 in the first): vector moves, not trips through LDS, as the
// lists take some hundred of them one after the other.
template <int O>
__device__ __forceinline__ uint32_t lp_xor_bits(uint32_t x) {
    const int v = (int)x;
    if constexpr (O == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false);
    if constexpr (O == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false);
    if constexpr (O == 4)  // (7 - i, then 3 - i within four)
        return (uint32_t)__builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false), 0x1B, 0xf, 0xf, false);
    if constexpr (O == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, false);
    if constexpr (O == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    }
    if constexpr (O == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
}
template <int O>
__device__ __forceinline__ float lp_xor(float x) { return __uint_as_float(lp_xor_bits<O>(__float_as_uint(x))); }
template <int O>
__device__ __forceinline__ int lp_xor(int x) { return (int)lp_xor_bits<O>((uint32_t)x); }
__device__ __forceinline__ uint32_t lp_before_lane(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x138, 0xf, 0xf, false);
}
__device__ __forceinline__ float lp_wave_max(float v) {
    v = fmaxf(v, lp_xor<1>(v));
    v = fmaxf(v, lp_xor<2>(v));
    v = fmaxf(v, lp_xor<4>(v));
    v = fmaxf(v, lp_xor<8>(v));
    v = fmaxf(v, lp_xor<16>(v));
    return fmaxf(v, lp_xor<32>(v));
}

// A candidate: value and index.  a before b: the larger value, the lower index among equal ones.
__device__ __forceinline__ bool lp_before(float av, int ai, float bv, int bi) { return av > bv || (av == bv && ai < bi); }

// A list over lanes: lane i the i-th candidate.
struct LpList {
    float v;
    int i;
};
template <int O>
__device__ __forceinline__ void lp_order(LpList& a) {  // the lane without bit O keeps the one that comes first
    const float v = lp_xor<O>(a.v);
    const int i = lp_xor<O>(a.i);
    if (lp_before(v, i, a.v, a.i) == !(threadIdx.x & O)) {
        a.v = v;
        a.i = i;
    }
}
// Lists of up to 32, one in each half of a wave: the 32 first of a list and another one, (rv, ri) from its end, sorted
static_assert(LOGP_MAX_TOP <= 32, "a list fits half a wave");
__device__ __forceinline__ void lp_merge(LpList& a, float rv, int ri) {
    if (lp_before(rv, ri, a.v, a.i)) {
        a.v = rv;
        a.i = ri;
    }
    lp_order<16>(a);
    lp_order<8>(a);
    lp_order<4>(a);
    lp_order<2>(a);
    lp_order<1>(a);
}
// and of the two halves' lists
__device__ __forceinline__ void lp_merge_halves(LpList& a) {
    lp_merge(a, __shfl_xor(a.v, 63, 64), __shfl_xor(a.i, 63, 64));
}
// A number that at least k lanes' values reach, close below the k-th largest of them (-inf if fewer than k are above): by halving
// an interval of the floats' order, which a count of lanes decides and scalar instructions carry.
__device__ __forceinline__ int lp_key(float v) {
    const int b = (int)__float_as_uint(v);
    return b ^ (b >> 31 & 0x7fffffff);
}
__device__ __forceinline__ float lp_kth(float v, int k) {
    const int key = lp_key(v == v ? v : LP_NONE);
    auto reach = [&](int t) { return __popcll(__ballot(key >= t)) >= k; };
    int lo = lp_key(LP_NONE), hi = __builtin_amdgcn_readfirstlane(lp_key(lp_wave_max(v == v ? v : LP_NONE)));  // (reached; by one lane)
    if (hi > lo + (1 << 25) && reach(hi - (1 << 25))) lo = hi - (1 << 25);  // (within some 16 times or 4 halvings of the largest)
#pragma unroll 1
    for (int i = 0; i < 12; ++i) {
        const int mid = lo + (int)(((uint32_t)hi - (uint32_t)lo) >> 1);
        if (reach(mid)) lo = mid;
        else hi = mid;
    }
    return __uint_as_float((uint32_t)(lo ^ (lo >> 31 & 0x7fffffff)));
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
// The 2048 logits of a row of V from `at` on, -inf behind its end.
template <bool BF16>
__device__ __forceinline__ void lp_load(const void* row, int at, int V, int lane, LpRaw<BF16>& r) {
    if (at + LP_SUB <= V) {
        if (BF16) {
            const uint16_t* p = static_cast<const uint16_t*>(row) + at;
#pragma unroll
            for (int j = 0; j < LP_PER / 8; ++j) {
                const LpH8 x = *reinterpret_cast<const LpH8*>(p + j * 512 + lane * 8);
#pragma unroll
                for (int i = 0; i < 4; ++i) r.w[4 * j + i] = x.v[2 * i] | (uint32_t)x.v[2 * i + 1] << 16;
            }
        } else {
            const float* p = static_cast<const float*>(row) + at;
#pragma unroll
            for (int j = 0; j < LP_PER / 4; ++j) {
                const LpF4 x = *reinterpret_cast<const LpF4*>(p + j * 256 + lane * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) r.w[4 * j + i] = __float_as_uint(x.v[i]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < LP_PER; ++i) {
            const int j = at + lp_index<BF16>(i, lane);
            if (BF16) {
                const uint32_t v = j < V ? static_cast<const uint16_t*>(row)[j] : 0xff80u;
                r.w[i / 2] = i % 2 ? r.w[i / 2] | v << 16 : v;
            } else {
                r.w[i] = j < V ? static_cast<const uint32_t*>(row)[j] : 0xff800000u;
            }
        }
    }
}
template <bool BF16>
__device__ __forceinline__ float lp_value(const LpRaw<BF16>& r, int e) {
    return BF16 ? (e & 1 ? bf_hi(r.w[e / 2]) : bf_lo(r.w[e / 2])) : __uint_as_float(r.w[e]);
}

template <bool BF16>
__device__ __forceinline__ float lp_most(const LpRaw<BF16>& r) {
    float m = lp_value<BF16>(r, 0);
#pragma unroll
    for (int e = 1; e < LP_PER; ++e) m = fmaxf(m, lp_value<BF16>(r, e));
    return m;
}

// The logit of a row's token, or NaN for a token outside the vocabulary.
template <bool BF16>
__device__ __forceinline__ float lp_token(const LogpArgs& a, int64_t row) {
    const int t = a.logprob ? a.tokens[row] : -1;
    if (t < 0 || t >= a.V) return __builtin_nanf("");
    const int64_t at = row * a.stride + t;
    return BF16 ? bf2f(static_cast<const uint16_t*>(a.logits)[at]) : static_cast<const float*>(a.logits)[at];
}
// A row's results from its joined state and list and its token's logit.
template <bool BF16>
__device__ __forceinline__ void lp_finish(const LogpArgs& a, int64_t row, const LpState& s, const LpList& list, float x) {
    const int lane = threadIdx.x & 63;
    const float ln = s.S == 0.0f ? 0.0f : logf(s.S);
    if (lane < a.top) {
        const bool some = list.v > LP_NONE;
        if (a.top_tokens) a.top_tokens[row * a.top + lane] = some ? list.i : -1;
        if (a.top_logprobs) a.top_logprobs[row * a.top + lane] = some ? (list.v - s.m) - ln : LP_NONE;
    }
    if (lane == 0) {
        if (a.entropy) a.entropy[row] = s.S == 0.0f ? 0.0f : ln - ieee_div(s.T, s.S);
        // (a row that is masked whole has no reference)
        if (a.logprob) a.logprob[row] = s.m == LP_NONE && s.S == 0.0f ? x : (x - s.m) - ln;
    }
}

// One block a segment of a row; its waves take every LP_WAVES-th 2048 logits of it.  Alone in its row it writes the results, else
// its state and list.
template <bool BF16, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void logprobs_kernel(LogpArgs a, int segs) {
    __shared__ float sv[LP_WAVES][32], sm[LP_WAVES][3], sf[LP_WAVES];
    __shared__ int si[LP_WAVES][32];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x / segs;
    const int seg = blockIdx.x % segs;
    const int subs = (a.V + LP_SUB - 1) / LP_SUB;
    const int s0 = (int)((int64_t)subs * seg / segs), s1 = (int)((int64_t)subs * (seg + 1) / segs);
    const void* p = BF16 ? (const void*)(static_cast<const uint16_t*>(a.logits) + row * a.stride)
                         : (const void*)(static_cast<const float*>(a.logits) + row * a.stride);
    LpState st{LP_NONE, 0.0f, 0.0f};
    LpList list{LP_NONE, 0x7fffffff};
    float floor = LP_NONE, most = LP_NONE;  // at least `top` logits of the segment reach floor; most: the lane's largest of the wave's part
    LpRaw<BF16> next;
    const float own = wave == 0 && segs == 1 ? lp_token<BF16>(a, row) : 0.0f;  // (requested before it is needed)
    if (s0 + wave < s1) lp_load<BF16>(p, (s0 + wave) * LP_SUB, a.V, lane, next);
    if (TOP) {
        // each of the waves' first parts has k lanes whose largest logit reaches its k-th largest, so `top` logits reach the least of these
        const int k = (a.top + min(LP_WAVES, s1 - s0) - 1) / min(LP_WAVES, s1 - s0);
        if (s0 + wave < s1) most = lp_most<BF16>(next);
        const float kth = lp_kth(most, k);
        if (lane == 0) sf[wave] = s0 + wave < s1 ? kth : -LP_NONE;
        __syncthreads();
        floor = fmaxf(fminf(fminf(sf[0], sf[1]), fminf(sf[2], sf[3])), -3.402823466e38f);  // (-inf is no candidate)
    }
    float last = floor;  // of the list, if it is full
    for (int s = s0 + wave; s < s1; s += LP_WAVES) {
        LpRaw<BF16> x = next;
        const int base = s * LP_SUB;
        if (s + LP_WAVES < s1) lp_load<BF16>(p, (s + LP_WAVES) * LP_SUB, a.V, lane, next);
        if (!TOP || s != s0 + wave) most = lp_most<BF16>(x);
        const float top = fmaxf(st.m, lp_wave_max(most));
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
            if (__any(most >= at)) {
#pragma unroll
                for (int e = 0; e < LP_PER; ++e) {
                    const float v = lp_value<BF16>(x, e);
                    unsigned long long hit = __ballot(v >= at);
                    while (hit) {
                        const int l = __ffsll(hit) - 1;
                        hit &= hit - 1;
                        const float cv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l));
                        const int ci = base + lp_index<BF16>(e, l);
                        const int pos = __popcll(__ballot(lp_before(list.v, list.i, cv, ci)));
                        if (pos < a.top) {
                            const float uv = __uint_as_float(lp_before_lane(__float_as_uint(list.v)));
                            const int ui = (int)lp_before_lane((uint32_t)list.i);
                            list.v = lane < pos ? list.v : lane == pos ? cv : uv;
                            list.i = lane < pos ? list.i : lane == pos ? ci : ui;
                            at = last = fmaxf(last, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(list.v), a.top - 1)));
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
    if (TOP && lane < 32) {
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
        static_assert(LP_WAVES == 4, "two lists a half");
        const int h = lane >> 5, i = lane & 31;
        list = LpList{sv[h][i], si[h][i]};
        lp_merge(list, sv[h + 2][31 - i], si[h + 2][31 - i]);
        lp_merge_halves(list);
    }
    if (segs == 1) {
        lp_finish<BF16>(a, row, sum, list, own);
        return;
    }
    float* part = static_cast<float*>(a.part) + (int64_t)blockIdx.x * lp_width(a.top);
    if (lane == 0) *reinterpret_cast<float4*>(part) = make_float4(sum.m, sum.S, sum.T, 0.0f);
    if (TOP && lane < a.top) {
        part[4 + lane] = list.v;
        reinterpret_cast<int*>(part)[4 + a.top + lane] = list.i;
    }
}

// One block a row: its segments' states and lists join, half a wave a list, then the halves and the waves.
constexpr int LP_JOIN_WAVES = 4;
template <bool BF16, bool TOP>
__global__ __launch_bounds__(64 * LP_JOIN_WAVES) void logprobs_join_kernel(LogpArgs a, int segs) {
    __shared__ float sv[LP_JOIN_WAVES][32];
    __shared__ int si[LP_JOIN_WAVES][32];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x;
    const int width = lp_width(a.top);
    const float* part = static_cast<const float*>(a.part) + row * segs * width;
    const float own = wave ? 0.0f : lp_token<BF16>(a, row);
    LpState st{LP_NONE, 0.0f, 0.0f};
    if (lane < segs) {
        const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)lane * width);
        st = LpState{x.x, x.y, x.z};
    }
    LpList list{LP_NONE, 0x7fffffff};
    if (TOP) {
        // a half's first list as it is, the others from their ends
        const int h = lane >> 5, i = lane & 31;
        for (int s = 2 * wave; s < segs; s += 2 * LP_JOIN_WAVES) {
            const bool first = s == 2 * wave;
            const int j = first ? i : 31 - i;
            float v = LP_NONE;
            int id = 0x7fffffff;
            if (s + h < segs && j < a.top) {
                const float* q = part + (int64_t)(s + h) * width + 4;
                v = q[j];
                id = reinterpret_cast<const int*>(q)[a.top + j];
            }
            if (first)
                list = LpList{v, id};
            else
                lp_merge(list, v, id);
        }
        lp_merge_halves(list);
        if (h == 0) {
            sv[wave][i] = list.v;
            si[wave][i] = list.i;
        }
        __syncthreads();
        if (wave) return;
        static_assert(LP_JOIN_WAVES == 4, "two lists a half");
        list = LpList{sv[h][i], si[h][i]};
        lp_merge(list, sv[h + 2][31 - i], si[h + 2][31 - i]);
        lp_merge_halves(list);
    }
    if (wave) return;
    lp_move(st, wave_max(st.m));
    st.S = wave_sum_fast(st.S);
    st.T = wave_sum_fast(st.T);
    lp_finish<BF16>(a, row, st, list, own);
}

// Segments of a row: until there are LP_BLOCKS_PER_CU, or every wave has one part.
int segments(const LogpArgs& a) {
    const int64_t subs = ((int64_t)a.V + LP_SUB - 1) / LP_SUB;
    const int64_t most = std::min<int64_t>((subs + LP_WAVES - 1) / LP_WAVES, LP_MAX_SEGS);
    return (int)std::max<int64_t>(1, std::min<int64_t>(most, (LP_BLOCKS_PER_CU * a.n_cu + a.n - 1) / a.n));
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
