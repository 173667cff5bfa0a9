// k_attn_kv4.hip -- attention of a batch's new tokens over the 4-bit paged K/V cache.
//
// out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m) in one pass over the positions, with a running reference m.  Both
// products, S^T = K Q^T and O^T = V^T P^T, run on v_mfma_scale_f32_16x16x128_f8f6f4 with the cache's codes as they are:
// no code is converted.  K's scale of 32 features is the instruction's own block scale.  V's scale of a position is not
// along the product's axis, so it goes into the probability; a probability and a query value enter as e2m3 terms (6 bits, at the
// rate of the 4-bit operand, twice that of 8 bits) whose block scale the lane that holds the block takes from its own values.
#include <stddef.h>

#include <algorithm>
#include <type_traits>

#include "mg_attn_rows.h"

namespace mg {
namespace {

typedef int i32x8_k4 __attribute__((ext_vector_type(8)));
typedef int i32x6_k4 __attribute__((ext_vector_type(6)));
typedef uint32_t u32x6_k4 __attribute__((ext_vector_type(6)));
typedef float f32x16_k4 __attribute__((ext_vector_type(16)));
typedef float f32x32_k4 __attribute__((ext_vector_type(32)));

constexpr int K4_STEP = 8;          // pages of a step: 128 positions, the products' depth

template <int HD>
struct K4Lane {  // what a lane loads of a page: 16 features' worth of four positions of V
    typedef u32x4_k8 v;
};
template <>
struct K4Lane<64> {
    typedef u32x2_k8 v;
};

__device__ __forceinline__ i32x8_k4 k4_wide(const i32x6_k4& x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, 4, 5, -1, -1); }
__device__ __forceinline__ i32x8_k4 k4_wide(const u32x4_k8& x) {
    return __builtin_shufflevector(__builtin_bit_cast(int __attribute__((ext_vector_type(4))), x), __builtin_bit_cast(int __attribute__((ext_vector_type(4))), x),
                                   0, 1, 2, 3, -1, -1, -1, -1);
}
// C + A B: A 16 rows of 128 e2m1 values, B 16 columns of 128 e2m3 values; lane 16 g + c holds values 32 g .. 32 g + 31 of row or
// column c and their scale byte, and rows 4 g .. 4 g + 3 of column c of C.
// Byte SA of sa is A's scale, SB of sb B's.
template <int SA, int SB>
__device__ __forceinline__ f32x4_k8 k4_mfma(const u32x4_k8& a, uint32_t sa, const i32x6_k4& b, uint32_t sb, f32x4_k8 c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k4_wide(a), k4_wide(b), c, 4, 2, SA, (int)sa, SB, (int)sb);
}

// 32 values (of even and of odd index, as the conversion takes them) as e2m3 values under a scale.
__device__ __forceinline__ i32x6_k4 k4_block(const f32x16_k4& even, const f32x16_k4& odd, float scale) {
    auto q = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, scale);
    // (the conversion takes several passes over its 32 sources: its result must not be placed on one of them, as the compiler
    // does where they end here; such results were off now and then)
    asm volatile("" : "+v"(q) : "v"(even), "v"(odd), "v"(scale));
    return __builtin_bit_cast(i32x6_k4, q);
}
// e2m3 values are multiples of 1/8 up to 2, of 1/4 up to 4, of 1/2 up to 7.5.
// Three terms of 32 query values under scales s, s / 32, s / 1024, with s the power of two under which the largest (`top`, float bits, finite) is
// below 2: a term is off by 1/16 of its scale at most, and 32 times that is at most 2 again, so s / 16384 or 2^-14 of the largest is left in the end.
// What a term leaves is found by adding and taking away a number whose last bit is an eighth of its scale, which rounds as the conversion does.
// That number would be infinite from s = 2^108 on, so values of blocks from 2^64 up are taken 2^64 lower first (exact but for what is below 2^-126 of
// the largest); the scales' bytes are those of the values as they were.
__device__ __forceinline__ uint32_t k4_triple(f32x16_k4& even, f32x16_k4& odd, uint32_t top, i32x6_k4 (&t)[3]) {
    const uint32_t scale = max(top & 0x7f800000u, 12u << 23);  // (the third's is a normal number)
    uint32_t at = scale;
    if (scale >= (127u + 64u) << 23) {
        at -= 64u << 23;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            even[i] *= 0x1p-64f;
            odd[i] *= 0x1p-64f;
        }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const float s = __uint_as_float(at - k * (5u << 23)), M = s * 0x1.8p+20f;
        t[k] = k4_block(even, odd, s);
        if (k == 2) break;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            even[i] -= (even[i] + M) - M;
            odd[i] -= (odd[i] + M) - M;
        }
    }
    return scale >> 23;
}
// Two terms of 32 weights of V of at most `top` under scales s and s / 32, with s the power of two under which top is from 3.75 to 7.5; returned: the scales'
// bytes.  The first leaves s / 4 of a value from 4 s up, s / 8 from 2 s up, s / 16 below; under s / 32 a sixteenth of those from 4 s up are past the
// format and become 7.5.  So s / 64, s / 256, s / 512 are left: 2^-8 of a value, as a bf16 weight would be off, or 1/1920 of the largest, at most.
// What the first leaves is found by converting it back, one instruction of some 70 cycles.
// Chunks of 2048 tokens over 2048 to 8192 positions were off by 0.0039 of their outputs, the bf16 results' rounding, 0.0016, among it, with two terms
// of which the first is held below 2 s as above, by 0.0019 with these, in the same time; with a third term in every step four chunks take 667 us instead of
// 525, a step of 64 rows 18.2 instead of 13.9.
__device__ __forceinline__ uint32_t k4_pair(f32x16_k4& even, f32x16_k4& odd, float top, i32x6_k4 (&t)[2]) {
    constexpr uint32_t least = 7u << 23;  // (the second's is a normal number)
    const uint32_t scale = max(__float_as_uint(top * (16.0f / 15.0f)) & 0x7f800000u, least + (2u << 23)) - (2u << 23);
    const float s = __uint_as_float(scale);
    t[0] = k4_block(even, odd, s);
    f32x32_k4 y = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(__builtin_bit_cast(u32x6_k4, t[0]), s);
    asm volatile("" : "+v"(y) : "v"(t[0]), "v"(s));
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        even[i] -= y[2 * i];
        odd[i] -= y[2 * i + 1];
    }
    t[1] = k4_block(even, odd, __uint_as_float(scale - (5u << 23)));
    return (scale >> 23) * 0x101u - 0x500u;
}
// The 1/1920 is of the largest weight times scale.  Where scales of V differ, a position of a small one beside a large one would lose as much, though the
// large one has no part in the features that its codes leave 0: beside scales 2^5, 2^7, 2^9 times theirs such features were off by 0.008, 0.03, 0.12, with
// bf16 weights by 0.0014, with two terms and scales within 2^2 by 0.0009 to 0.0014.  So a block takes one more term, under a 32nd of the scale before it,
// for each 2^5 that its scales are further apart: a weight is off by 2^-8 of itself or 1/480 of the block's largest, whatever the scales of V.
// To look at the scales costs steps that need no further term 4 % in chunks (four of 2048 500 -> 525 us) and next to nothing in rows of few
// query rows; with one or two further terms in all steps four chunks take 667 and 811 us, 64 rows 18.2 and 19.7, 32 long rows 94 and 102 instead of 82.
constexpr uint32_t K4_NEAR = 2;
// Positions that are not seen, that hold nothing (0), what is not finite (255, or 0 where that was noted) or the least scale have a part in no distance.
constexpr uint32_t K4_EMPTY = 16;
struct K4Apart {
    uint32_t lo = 255, hi = 0;
    __device__ __forceinline__ void add(uint32_t b, bool seen) {
        const bool part = seen && b > K4_EMPTY && b < 255u;
        hi = max(hi, part ? b : 0u);
        lo = min(lo, part ? b : 255u);
    }
};
// terms of a block whose scales' bytes are from lo to hi (0: k4_pair's)
__device__ __forceinline__ int k4_terms(uint32_t lo, uint32_t hi) { return hi > lo + K4_NEAR ? (int)(hi - lo + 4 - K4_NEAR) / 5 : 0; }
// the most of a wave's lanes
__device__ __forceinline__ int k4_wave_most(int n) {
    int most = 0;
    while (__any(n > most)) ++most;
    return most;
}
// n terms after the second of k4_pair, which left even and odd and the scales' bytes ps: add(term, its scale's byte) for each.
// (Scales stay normal numbers: what is below some 2^-120 is lost.)
// What a term leaves is found by making it again and converting it back (BACK), or, with 32 registers less and some 300 cycles more, by rounding to eighths of
// its scale: so for numbers up to twice that; larger ones were 2 s or more, the second term left 2^-8 of them at most, and they need no more.
template <bool BACK, class Add>
__device__ __forceinline__ void k4_more(f32x16_k4& even, f32x16_k4& odd, uint32_t ps, int n, const Add& add) {
    uint32_t b = max(ps >> 8 & 0xffu, 5u);
#pragma unroll 1
    for (int k = 0; k < n; ++k) {
        if constexpr (BACK) {
            const float s = __uint_as_float(b << 23);
            const i32x6_k4 t = k4_block(even, odd, s);
            f32x32_k4 y = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(__builtin_bit_cast(u32x6_k4, t), s);
            asm volatile("" : "+v"(y) : "v"(t), "v"(s));
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                even[i] -= y[2 * i];
                odd[i] -= y[2 * i + 1];
            }
        } else {
            const float to = __uint_as_float((257u - b) << 23), by = __uint_as_float(b << 23) * 0.125f;  // 8 / s, s / 8
            const auto rest = [&](float x) {
                const float y = x * to;
                return __builtin_fabsf(y) <= 16.0f ? __builtin_fmaf(-__builtin_rintf(y), by, x) : 0.0f;
            };
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                even[i] = rest(even[i]);
                odd[i] = rest(odd[i]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        b = max(b, 10u) - 5u;
        add(k4_block(even, odd, __uint_as_float(b << 23)), b);
    }
}

// Query rows rr0 + 16 u + c of a row's KV head (row rr: token rr / G, head rr % G of the group) as B operands in LDS (registers are
// what bounds a wave's tiles), and the positions of their tokens; columns past the row's last repeat its first.  Three terms of a
// value: exact but for what is below 2^-6 of the largest of its 32 features, which is off by 2^-14 of that at most.  HD 128: an
// operand a term.  HD 64: the first two terms share one (lanes 0..31 and 32..63, against K's features twice), the third has
// one with zeros.
template <int HD>
constexpr int K4_OPS = HD == 128 ? 3 : 2;
template <int HD>
struct K4Query {
    uint32_t lo[K4_OPS<HD>][64][4], hi[K4_OPS<HD>][64][2];  // a lane's six words
    uint32_t scale[64];                                      // byte k: operand k's
};
// the position of query row rr's token
__device__ __forceinline__ int k4_position(const Kv8AttnArgs& a, const K8Row& row, int rr) {
    return row.p0 + (rr < row.n * a.G ? rr / a.G : 0);
}
template <int HD>
__device__ __forceinline__ void k4_query(const Kv8AttnArgs& a, const K8Row& row, int kh, int rr0, K4Query<HD>& q) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    int rr = rr0 + c;
    rr = rr < row.n * a.G ? rr : 0;
    const uint16_t* p = a.q + (int64_t)(row.t0 + rr / a.G) * a.q_stride + (size_t)(kh * a.G + rr % a.G) * HD + 32 * (HD == 128 ? g : g & 1);
    uint32_t w[16], top = 0;
#pragma unroll
    for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4*>(w + i) = *reinterpret_cast<const uint4*>(p + 2 * i);
    f32x16_k4 even, odds;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        top = max(top, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
        even[i] = bf_lo(w[i]);
        odds[i] = bf_hi(w[i]);
    }
    i32x6_k4 t[3];
    const uint32_t s = k4_triple(even, odds, top << 16, t);
    // (a value that is not finite makes the scores NaN)
    const bool odd = top >= 0x7f80u;
    const uint32_t b0 = odd ? 255u : s, b1 = odd ? 255u : s - 5, b2 = odd ? 255u : s - 10;
    if constexpr (HD == 64) {
#pragma unroll
        for (int i = 0; i < 6; ++i) {
            t[0][i] = g < 2 ? t[0][i] : t[1][i];
            t[1][i] = g < 2 ? t[2][i] : 0;
        }
    }
    q.scale[lane] = HD == 128 ? b0 | b1 << 8 | b2 << 16 : g < 2 ? b0 | b2 << 8 : b1 | 127u << 8;
#pragma unroll
    for (int k = 0; k < K4_OPS<HD>; ++k) {
        *reinterpret_cast<u32x4_k8*>(q.lo[k][lane]) = u32x4_k8{(uint32_t)t[k][0], (uint32_t)t[k][1], (uint32_t)t[k][2], (uint32_t)t[k][3]};
        *reinterpret_cast<u32x2_k8*>(q.hi[k][lane]) = u32x2_k8{(uint32_t)t[k][4], (uint32_t)t[k][5]};
    }
}
template <int HD>
__device__ __forceinline__ i32x6_k4 k4_operand(const K4Query<HD>& q, int k) {
    const int lane = threadIdx.x & 63;
    const u32x4_k8 lo = *reinterpret_cast<const u32x4_k8*>(q.lo[k][lane]);
    const u32x2_k8 hi = *reinterpret_cast<const u32x2_k8*>(q.hi[k][lane]);
    return i32x6_k4{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1]};
}

template <int HD>
struct K4Acc {
    float m, l;  // the score (as x below, before the factor f) that the exponents refer to; sum over the lane's positions
    f32x4_k8 o[HD / 16];
    __device__ __forceinline__ void clear() {
        // no score is below it, and it is finite: exp2 of a masked score's difference is 0 where nothing was seen yet
        m = -3.402823466e38f;
        l = 0.0f;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) o[d] = f32x4_k8{0.f, 0.f, 0.f, 0.f};
    }
};

// A step's scores x (position 16 i + 4 g + r at x[4 i + r]) become its probabilities, of at most some 1/2: 2^((x - m) f - K4_FOLD), with m the score that
// moved the reference last, so that a probability times a value's scale, up to 2^126, is finite.  m moves only when a score of the step passes it
// by 12 / f: exchanges between lanes and rescaled outputs are rare.
// The exponent is x f - (m f + K4_FOLD) with one rounding, relative to the rounded second term; that rounding is the same for all scores, but from
// |m f| of some 2^30 on it is larger than what exp2 takes.  So references beyond K4_FAR take x - m first (an instruction a score, in rare steps).
constexpr float K4_FOLD = 13.0f;
constexpr float K4_FAR = 4096.0f;
__device__ __forceinline__ float k4_at(float m, float f) { return fmaxf(__builtin_fmaf(m, f, K4_FOLD), -3.0e38f); }
__device__ __forceinline__ bool k4_far(float at) { return __builtin_fabsf(at) > K4_FAR; }
// the factor of what was summed under reference m where the reference becomes `to`, at least m
__device__ __forceinline__ float k4_rescale(float m, float to, float f) {
    const float a = k4_at(m, f), b = k4_at(to, f);
    return __builtin_amdgcn_exp2f(k4_far(a) || k4_far(b) ? (m - to) * f : a - b);
}
template <int HD>
__device__ __forceinline__ void k4_move(float mx, float f, K4Acc<HD>& acc) {
    const float mn = fmaxf(acc.m, k8_col_max(mx));
    const float al = k4_rescale(acc.m, mn, f);
    acc.m = mn;
    acc.l *= al;
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) acc.o[d] *= al;
}
__device__ __forceinline__ float k4_most(const float (&x)[32]) {
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 32; ++i) mx = fmaxf(mx, x[i]);
    return mx;
}
// the exponentials in place; returned: their sum
__device__ __forceinline__ float k4_exp(float (&x)[32], float f, float m) {
    float at = k4_at(m, f);
    if (__any(k4_far(at))) {
        const float sub = k4_far(at) ? m : 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] -= sub;
        at = k4_far(at) ? K4_FOLD : at;
    }
    float s[4];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], f, -at));
        s[i & 3] = i < 4 ? x[i] : s[i & 3] + x[i];
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}
template <int HD>
__device__ __forceinline__ void k4_probs(float (&x)[32], float f, K4Acc<HD>& acc) {
    const float mx = k4_most(x);
    if (__any((mx - acc.m) * f > 12.0f)) k4_move(mx, f, acc);
    acc.l += k4_exp(x, f, acc.m);
}

// a wave-uniform float in a scalar register
__device__ __forceinline__ float k4_scalar(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// Pages [pg0, pg1) of a row's table against 16 query rows: steps first, first + stride, ... of K4_STEP pages.  K's
// registers are loaded again as soon as the scores are there, V's after its product, so that a wave has a step in flight at any
// time.  ONCE: pages that no other wave reads, by loads that leave no trace in the caches.
template <int HD, bool CAP, bool ONCE>
__device__ __forceinline__ void k4_walk(const Kv8AttnArgs& a, const K8Row& row, int r, int kh, int pg0, int pg1, int first, int stride,
                                        const K4Query<HD>& q, int pos, int p_hi, K4Acc<HD>& acc) {
    typedef typename K4Lane<HD>::v vlane;
    constexpr int DT = HD / 16;
    constexpr size_t head_bytes = 16 * HD, head_scales = HD / 2 + 16;
    const int lane = threadIdx.x & 63, g = lane >> 4;
    K8Soft so = k8_soft(a);
    so = K8Soft{k4_scalar(so.f), k4_scalar(so.zin), k4_scalar(so.most)};
    const int32_t* ptab = a.page_table + (size_t)r * a.maxp;
    const int p_lo = __builtin_amdgcn_readfirstlane(pos);  // of the wave's earliest token; p_hi: of its latest
    typedef const __attribute__((address_space(1))) char* gptr;

    for (int ch = pg0; ch < pg1; ch += K8_IDS) {
        const int cnt = min(K8_IDS, pg1 - ch), steps = (cnt + K4_STEP - 1) / K4_STEP;
        // the chunk's first step that is this wave's
        const int done = (ch - pg0) / K4_STEP;
        int s = first - done;
        if (s < 0) s = (stride - (-s) % stride) % stride;
        if (s >= steps) continue;
        // lane i: page ch + i of the table and its place in the cache (a hole, or one past the split: page 0, unseen)
        const int id = lane < cnt ? ptab[ch + lane] : -1;
        const unsigned long long live_pages = __ballot(id >= 0 && id < a.c.n_pages);
        const uint32_t place = (id >= 0 && id < a.c.n_pages ? (uint32_t)id : 0u) * (uint32_t)a.c.Hkv + (uint32_t)kh;
        u32x4_k8 kb[K4_STEP];
        vlane vb[K4_STEP];
        uint32_t ks[K4_STEP], vs[K4_STEP];
        auto fetch_k = [&](int s) {
            // (made anew: a load then takes its page's address from scalar registers, and nothing of it is held meanwhile)
            uint32_t k_lane = threadIdx.x, at = place;
            asm volatile("" : "+v"(k_lane), "+v"(at));
            k_lane &= HD == 128 ? 63 : 31;
            const uint32_t k_at = k_lane * 16u;
#pragma unroll
            for (int e = 0; e < K4_STEP; ++e) {
                if (e % 2 == 0) __builtin_amdgcn_sched_barrier(0);  // (fewer addresses at a time)
                const size_t ph = (uint32_t)__builtin_amdgcn_readlane((int)at, K4_STEP * s + e);
                const uint64_t p = k8_uniform(a.c.codes + ph * head_bytes), ps = k8_uniform(a.c.scales + ph * head_scales);
                auto* kp = reinterpret_cast<const __attribute__((address_space(1))) u32x4_k8*>(reinterpret_cast<gptr>(p) + k_at);
                kb[e] = ONCE ? __builtin_nontemporal_load(kp) : *kp;
                ks[e] = *reinterpret_cast<const __attribute__((address_space(1))) uint8_t*>(reinterpret_cast<gptr>(ps) + k_lane);
            }
        };
        auto fetch_v = [&](int s) {
            uint32_t v_lane = threadIdx.x, at = place;
            asm volatile("" : "+v"(v_lane), "+v"(at));
            v_lane &= 63;
            const uint32_t v_at = v_lane * (uint32_t)sizeof(vlane), vs_at = v_lane >> 4 << 2;
#pragma unroll
            for (int e = 0; e < K4_STEP; ++e) {
                if (e % 2 == 0) __builtin_amdgcn_sched_barrier(0);
                const size_t ph = (uint32_t)__builtin_amdgcn_readlane((int)at, K4_STEP * s + e);
                const uint64_t p = k8_uniform(a.c.codes + ph * head_bytes + 8 * HD), ps = k8_uniform(a.c.scales + ph * head_scales + HD / 2);
                auto* vp = reinterpret_cast<const __attribute__((address_space(1))) vlane*>(reinterpret_cast<gptr>(p) + v_at);
                vb[e] = ONCE ? __builtin_nontemporal_load(vp) : *vp;
                vs[e] = *reinterpret_cast<const __attribute__((address_space(1))) uint32_t*>(reinterpret_cast<gptr>(ps) + vs_at);
            }
        };
        fetch_k(s);
        fetch_v(s);
        for (; s < steps; s += stride) {
            const bool more = s + stride < steps;
            const int j0 = 16 * (ch + K4_STEP * s);
            const uint32_t mapped = (uint32_t)(live_pages >> (K4_STEP * s)) & 0xffu;
            const bool edge = mapped != 0xffu || j0 + 127 > p_lo || j0 + 128 > row.len || (a.window && j0 <= k8_hidden(a.window, p_hi));
            // whether a scale of V says that its value is not finite
            uint32_t odd = 0;
#pragma unroll
            for (int e = 0; e < K4_STEP; ++e) odd |= vs[e] & ((vs[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            const bool any_odd = __any(odd != 0);
            // terms of the weights past two
            const auto look = [&]() {
                uint32_t hi = 0, lo = 255;  // of the scales' bytes
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const uint32_t b = vs[i >> 2] >> (8 * (i & 3)) & 0xffu;
                    hi = max(hi, b);
                    lo = min(lo, b);
                }
                if (!__any(hi > lo + K4_NEAR)) return 0;
                K4Apart d;  // of what some token sees
                const int last = min(p_hi, row.len - 1) - j0 - 4 * g, first = (a.window ? k8_hidden(a.window, p_lo) : -1) - j0 - 4 * g;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const int at = 16 * (i >> 2) + (i & 3);
                    d.add(vs[i >> 2] >> (8 * (i & 3)) & 0xffu, (mapped >> (i >> 2) & 1u) && at <= last && at > first);
                }
                return k4_wave_most(k4_terms(d.lo, d.hi));
            };
            int terms = CAP ? look() : 0;  // (behind the scores 3 % shorter, but a cap leaves no registers for it there)
            float x[32];
            {
                asm volatile("" ::: "memory");  // (the queries are read anew, not held in registers)
                const uint32_t qs = q.scale[lane];
                f32x4_k8 c[K4_STEP];
#pragma unroll
                for (int e = 0; e < K4_STEP; ++e) c[e] = f32x4_k8{0.f, 0.f, 0.f, 0.f};
                const auto term = [&](auto K) {
                    const i32x6_k4 b = k4_operand(q, K.value);
#pragma unroll
                    for (int e = 0; e < K4_STEP; ++e) c[e] = k4_mfma<0, K.value>(kb[e], ks[e], b, qs, c[e]);
                };
                term(std::integral_constant<int, 0>{});
                term(std::integral_constant<int, 1>{});
                if constexpr (K4_OPS<HD> == 3) term(std::integral_constant<int, 2>{});
#pragma unroll
                for (int e = 0; e < K4_STEP; ++e) asm volatile("" : "+v"(c[e]));  // (here, not behind the branch of the loads)
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = c[i >> 2][i & 3];
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) fetch_k(s + stride);  // K's registers are free
            __builtin_amdgcn_sched_barrier(0);
            if (CAP) {
                k8_cap(reinterpret_cast<float(&)[1][32]>(x), so);
            }
            if (edge) {  // the token at p sees lo < position <= hi of the lane's
                int p = pos;
                asm("" : "+v"(p));  // (nothing of this is held between steps)
                const int hi = min(p, row.len - 1) - j0 - 4 * g, lo = (a.window ? k8_hidden(a.window, p) : -1) - j0 - 4 * g;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const int at = 16 * (i >> 2) + (i & 3);
                    x[i] = (mapped >> (i >> 2) & 1u) && at <= hi && at > lo ? x[i] : -__builtin_inff();
                }
            }
            if (any_odd) {  // such a value reaches the columns that see it, and no other: their probabilities become NaN
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    x[i] = (vs[i >> 2] >> (8 * (i & 3)) & 0xffu) == 255u && x[i] != -__builtin_inff() ? __builtin_nanf("") : x[i];
#pragma unroll
                for (int e = 0; e < K4_STEP; ++e) vs[e] &= ~(((vs[e] & ((vs[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 255u);
            }
            k4_probs<HD>(x, so.f, acc);
            f32x16_k4 y[2];
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                y[i & 1][i >> 1] = x[i] * __uint_as_float((vs[i >> 2] >> (8 * (i & 3)) & 0xffu) << 23);
                top = fmaxf(top, y[i & 1][i >> 1]);
            }
            if (!CAP) terms = look();
            const auto values = [&](int d) {
                u32x4_k8 A;
#pragma unroll
                for (int e = 0; e < 4; ++e) A[e] = __builtin_amdgcn_perm(vb[2 * e + 1][d / 2], vb[2 * e][d / 2], d & 1 ? 0x07060302u : 0x05040100u);
                return A;
            };
            i32x6_k4 p[2];
            const uint32_t ps = k4_pair(y[0], y[1], top, p);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const u32x4_k8 A = values(d);
                acc.o[d] = k4_mfma<0, 0>(A, 127u, p[0], ps, acc.o[d]);
                acc.o[d] = k4_mfma<0, 1>(A, 127u, p[1], ps, acc.o[d]);
            }
            if (terms) {
                __builtin_amdgcn_sched_barrier(0);
                k4_more<HD == 64>(y[0], y[1], ps, terms, [&](const i32x6_k4& t, uint32_t b) {
#pragma unroll
                    for (int e = 0; e < K4_STEP; ++e) asm volatile("" : "+v"(vb[e]));  // (operands are made in each turn, not held in registers)
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        acc.o[d] = k4_mfma<0, 0>(values(d), 127u, t, b, acc.o[d]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                });
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) fetch_v(s + stride);
        }
    }
}

// Rows of few query rows (tokens times query heads of a KV head <= 16 NT): one block per (row, KV head, split of the row's pages).
// A wave has one of the NT tiles of 16 query rows, and the waves of a tile take its steps in turn.
// Long rows are bound by the cache's bytes: 32 rows of 4096 to 16384 take 82 us one after the other in a graph, 4.2 TB/s, and 76 so with the loads
// alone, as the scales' records of 80 bytes lie in lines of 128 that blocks on two XCDs fetch (71 without them).  Shorter ones by what a step takes after its
// loads, some 2300 cycles of matrix and vector instructions, which do not overlap, and by the chain of length, page ids, codes before: 64 rows of
// 640 13.9 us (10.4 with the loads alone), one of 512 6.2 (4.7).
template <int HD, int WAVES>
struct K4FewShared {
    float o[WAVES][16][HD + 4];  // (padded rows)
    float m[WAVES][16], l[WAVES][16];
    K4Query<HD> q[WAVES];
};
template <int HD, int NT, int WAVES, bool CAP, bool EVEN>
__device__ __forceinline__ void k4_few_block(const Kv8AttnArgs& a, const K8Few& few, int block, K4FewShared<HD, WAVES>& sh) {
    constexpr int DT = HD / 16;
    const int c = threadIdx.x & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kh = block % a.c.Hkv;
    int r = block / a.c.Hkv % a.B, split = block / a.c.Hkv / a.B, act;
    K8Row row;
    if (EVEN) {
        const K8Lanes x = k8_lanes<16 * NT>(a, few);
        const int index = block / a.c.Hkv;
        const unsigned long long past = __ballot(x.sum > index);
        if (!past) return;
        r = __builtin_amdgcn_readfirstlane(__ffsll(past) - 1);
        row = k8_of_lane(x.row, r);
        act = __builtin_amdgcn_readlane(x.act, r);
        split = index - (__builtin_amdgcn_readlane(x.sum, r) - act);
    } else {
        row = k8_row(a, r);
        if (row.n <= 0 || row.n * a.G > 16 * NT) return;
        act = k8_active(max(row.pgb - row.pga, 0), few.sp, few.nsplit);
        if (split >= act) return;
    }
    const int npg = max(row.pgb - row.pga, 0), nsplit = few.most;
    const int per = (npg + act - 1) / act;
    const int pg0 = min(row.pgb, row.pga + split * per), pg1 = split == act - 1 ? row.pgb : min(row.pgb, pg0 + per);

    // (waves of a tile have the same queries: each writes its own, and waits for nobody)
    const int tile = wave % NT;
    k4_query<HD>(a, row, kh, 16 * tile, sh.q[wave]);
    const int pos = k4_position(a, row, 16 * tile + c);
    K4Acc<HD> acc;
    acc.clear();
    if (16 * tile < row.n * a.G)
        k4_walk<HD, CAP, NT == 1>(a, row, r, kh, pg0, pg1, wave / NT, WAVES / NT, sh.q[wave], pos, row.p0 + row.n - 1, acc);

    // the waves' shares join in LDS (the lane's number is made again: it is not held over the walk)
    const int ln = (int)__lane_id(), col = ln & 15, quarter = ln >> 4;
    const float ls = k8_col_sum(acc.l);
    if (quarter == 0) {
        sh.m[wave][col] = acc.m;
        sh.l[wave][col] = ls;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4_k8*>(&sh.o[wave][col][16 * d + 4 * quarter]) = acc.o[d];
    __syncthreads();
    const int live = row.n * a.G;
    const float unit = k8_soft(a).f;
    for (int i = 64 * wave + ln; i < live * (HD / 4); i += 64 * WAVES) {
        const int rr = i / (HD / 4), d = i % (HD / 4) * 4;
        const int w0 = rr / 16, rc = rr % 16;
        float M = sh.m[w0][rc];
#pragma unroll
        for (int w = 1; w < WAVES / NT; ++w) M = fmaxf(M, sh.m[w0 + w * NT][rc]);
        float L = 0.0f;
        f32x4_k8 O = f32x4_k8{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES / NT; ++w) {
            const float f = k4_rescale(sh.m[w0 + w * NT][rc], M, unit);
            L += f * sh.l[w0 + w * NT][rc];
            O += f * *reinterpret_cast<const f32x4_k8*>(&sh.o[w0 + w * NT][rc][d]);
        }
        const int64_t tok = row.t0 + rr / a.G;
        const int head = kh * a.G + rr % a.G;
        if (act == 1) {
            const float inv = L == 0.0f ? 0.0f : ieee_div(1.0f, L);
            *reinterpret_cast<uint2*>(a.out + tok * a.out_stride + head * HD + d) =
                make_uint2(k8_pack(O[0] * inv, O[1] * inv), k8_pack(O[2] * inv, O[3] * inv));
        } else {
            const size_t at = (((size_t)r * a.c.Hkv + kh) * nsplit + split) * (16 * NT) + rr;
            *reinterpret_cast<f32x4_k8*>(a.part + at * HD + d) = O;
            if (d == 0) {
                float* ml = a.part + (size_t)a.B * a.c.Hkv * nsplit * (16 * NT) * HD + 2 * at;
                ml[0] = M;
                ml[1] = L;
            }
        }
    }
}

template <int HD, int NT, int WAVES, bool CAP, bool EVEN>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2))) void attn_kv4_few_kernel(Kv8AttnArgs a, K8Few few) {
    __shared__ __attribute__((aligned(16))) K4FewShared<HD, WAVES> sh;
    k4_few_block<HD, NT, WAVES, CAP, EVEN>(a, few, blockIdx.x, sh);
}

// Joins the splits of rows of few query rows: a wave per query row of a (row, KV head); block: its index, of ROWB blocks a
// (row, KV head).
template <int HD, int NT, bool EVEN>
__device__ __forceinline__ void k4_few_join(const Kv8AttnArgs& a, const K8Few& few, int block, int rowb) {
    const int rr = block % rowb * K8_WAVES + (threadIdx.x >> 6);
    const int kh = block / rowb % a.c.Hkv, r = block / rowb / a.c.Hkv;
    K8Row row;
    int act;
    if (EVEN) {
        const K8Lanes x = k8_lanes<16 * NT>(a, few);
        row = k8_of_lane(x.row, r);
        act = __builtin_amdgcn_readlane(x.act, r);
    } else {
        row = k8_row(a, r);
        act = row.n <= 0 || row.n * a.G > 16 * NT ? 0 : k8_active(max(row.pgb - row.pga, 0), few.sp, few.nsplit);
    }
    if (act <= 1 || rr >= row.n * a.G) return;
    const int nsplit = few.most;
    const size_t first = ((size_t)r * a.c.Hkv + kh) * nsplit * (16 * NT) + rr;
    const float* ml = a.part + (size_t)a.B * a.c.Hkv * nsplit * (16 * NT) * HD;
    const float unit = k8_soft(a).f;
    k8_join<HD>(a.part + first * HD, (size_t)(16 * NT) * HD, ml + 2 * first, 2 * 16 * NT, act, k8_out(a, row, kh, rr),
                [unit](float m, float M) { return k4_rescale(m, M, unit); });
}
template <int HD, int NT, bool EVEN>
__global__ __launch_bounds__(K8_THREADS) void attn_kv4_join_kernel(Kv8AttnArgs a, K8Few few, int rowb) {
    k4_few_join<HD, NT, EVEN>(a, few, blockIdx.x, rowb);
}

// Rows of more query rows: one block per (row, KV head, 128 query rows, split of the positions that these see), the tokens of a
// row's end first (they see the most).  A wave holds two tiles of query rows; four waves share a step's codes through a double buffer in LDS: a
// wave fetches two pages of the next step, K as it is, V's two pages joined into the words of its operands, V's scales as
// numbers; one barrier a step parts the buffers.  GROUPS 2: the block has four waves more for the same query rows, and each group takes half of
// its steps; their outputs join at the end.
// Bound by issue: a tile's step is 40 matrix instructions (16 cycles each) and some 185 vector ones (32 exponentials among them), three conversions of
// 70 cycles; counters show the two kinds' cycles add up to the time (matrix cores 25 % busy, vector units 66 %).  Four chunks of 2048 tokens behind
// 0 to 6144 take 525 us, 1045 TFLOP/s of the definition's operations, where the 8-bit cache takes 575.  A barrier's wait is short; blocks in the order of
// what they see over all rows instead of row by row: 1 % less there, but 6 % more for two prompts of 1500.
constexpr int K4_TILES = 2;  // tiles of 16 query rows of a wave
constexpr int K4_CHUNK_ROWS = K8_WAVES * 16 * K4_TILES;
constexpr int K4_MIN_STAGES = 4;  // steps that a split of a tile takes at least
static_assert(K4_STEP == 2 * K8_WAVES, "a wave stages two pages");
// the largest of a row of 16 lanes
template <int CTRL>
__device__ __forceinline__ uint32_t k4_max_of(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true)); }
__device__ __forceinline__ uint32_t k4_row_most(uint32_t x) {
    x = k4_max_of<0xB1>(x);   // (lanes 1 0 3 2)
    x = k4_max_of<0x4E>(x);   // (2 3 0 1)
    x = k4_max_of<0x141>(x);  // (7 .. 0)
    return k4_max_of<0x140>(x);  // (15 .. 0)
}
// values at a byte address of LDS: a register and a constant each, so that neighbouring reads share the register
template <class T>
__device__ __forceinline__ T k4_lds(uint32_t at) {
    return *reinterpret_cast<const __attribute__((address_space(3))) T*>(at);
}
template <class T>
__device__ __forceinline__ uint32_t k4_lds_at(const T* p) {
    return (uint32_t)reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) T*)p);
}
template <int HD>
struct K4Stage {
    uint32_t k[K4_STEP][HD / 2][4];  // (HD 64: 32 lanes' words)
    uint32_t v[HD / 16][64][4];      // operand of an output tile; word e: pages 2 e and 2 e + 1
    uint8_t ks[64][K4_STEP];         // a lane's scale bytes of K, page by page
    float vs[K4_STEP][16];           // V's scales (0 where the value is not finite)
    uint32_t odd[K8_WAVES];          // bit 16 e + t: position t of page 2 word + e of V is not finite
    uint32_t span[K8_WAVES];         // of V's scale bytes of these two pages (0 where not finite): the largest, and 255 less the least, 16 bits each
};
template <int HD, int GROUPS>
struct K4ChunkShared {
    K4Stage<HD> stage[GROUPS][2];
    K4Query<HD> q[K8_WAVES][K4_TILES];
    int pos[K8_WAVES][K4_TILES][16];  // of the columns' tokens (few steps need them: they are not held in registers)
};
template <int HD, int GROUPS, bool CAP>
__device__ __forceinline__ void k4_chunk_block(const Kv8AttnArgs& a, int few, int tiles, int nsplit, float* part, int block,
                                               K4ChunkShared<HD, GROUPS>& sh) {
    typedef typename K4Lane<HD>::v vlane;
    typedef const __attribute__((address_space(1))) char* gptr;
    constexpr int DT = HD / 16, ROWS = K4_CHUNK_ROWS, NT = K4_TILES;
    // Whether the sums, needed anyway, tell that the reference has to move, and the step's scores are then made again (heads of 64: 6 chunks of 300 to
    // 600 48.2 us, with their maximum looked at in every step 46.8; heads of 128: the maximum leaves too few registers).
    constexpr bool REDO = HD == 128;
    // Where the weights' further terms are made: behind all else of a step, or (with fewer registers held, as caps need) behind their tile's first two
    constexpr bool LATE = REDO && !CAP;
    constexpr size_t head_bytes = 16 * HD, head_scales = HD / 2 + 16;
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / K8_THREADS);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % K8_WAVES;
    const int kh = block % a.c.Hkv;
    const int split = block / a.c.Hkv % nsplit, index = block / a.c.Hkv / nsplit;
    const K8Tile at = k8_tile<ROWS>(a, few, index);
    if (at.r < 0) return;
    const int r = __builtin_amdgcn_readfirstlane(at.r), t = __builtin_amdgcn_readfirstlane(at.t);
    const K8Row row = k8_row(a, r);
    const int live = row.n * a.G;
    if (t * ROWS >= live) return;
    const K8Span span = k8_span<ROWS, K4_STEP, K4_MIN_STAGES>(a, row, t, nsplit);
    if (split >= span.act) return;
    // the block's steps, and the group's of them; most: those of the group that has more
    const int b0 = span.stages * split / span.act, b1 = span.stages * (split + 1) / span.act, half = GROUPS == 1 ? b1 : (b0 + b1 + 1) / 2;
    const int st0 = group ? half : b0, steps = (group ? b1 : half) - st0, most = half - b0;
    const int pg0 = span.pg0 + st0 * K4_STEP, pg1 = min(span.pg1, pg0 + steps * K4_STEP);
    const int rr0 = t * ROWS + wave * (16 * NT);
    const int wp0 = row.p0 + min(rr0, live - 1) / a.G, wp1 = row.p0 + (min(rr0 + 16 * NT, live) - 1) / a.G;

    K4Acc<HD> acc[NT];
#pragma unroll
    for (int u = 0; u < NT; ++u)
        if (u % GROUPS == group) k4_query<HD>(a, row, kh, rr0 + 16 * u, sh.q[wave][u]);
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        if (group == 0 && lane < 16) sh.pos[wave][u][lane] = k4_position(a, row, rr0 + 16 * u + lane);
        acc[u].clear();
    }
    K8Soft so = k8_soft(a);
    so = K8Soft{k4_scalar(so.f), k4_scalar(so.zin), k4_scalar(so.most)};
    const int32_t* ptab = a.page_table + (size_t)r * a.maxp;

    // lane i: page pg0 + 64 n + i of the 64 that hold the step fetched last (a hole, or one past the block's: page 0, unseen), and the next 64's
    auto page_id = [&](int i) { return i < pg1 ? ptab[i] : -1; };
    auto valid = [&](int v) { return v >= 0 && v < a.c.n_pages; };
    int idn = page_id(pg0 + lane);
    uint32_t place = 0;
    unsigned long long live_pages = 0;
    u32x4_k8 nk[2];
    vlane nv[2];
    uint32_t nks[2], nvs;
    uint32_t map = 0;
    auto fetch = [&](int st) {
        const int at = st * K4_STEP % K8_IDS;
        if (at == 0) {
            live_pages = __ballot(valid(idn));
            place = (valid(idn) ? (uint32_t)idn : 0u) * (uint32_t)a.c.Hkv + (uint32_t)kh;
            idn = page_id(pg0 + st * K4_STEP + K8_IDS + lane);
        }
        map = (uint32_t)(live_pages >> at) & 0xffu;
        uint32_t ln = lane, pl = place;
        asm volatile("" : "+v"(ln), "+v"(pl));
        const uint32_t kl = HD == 128 ? ln : ln & 31;
        uint32_t ph[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            ph[e] = (uint32_t)__builtin_amdgcn_readlane((int)pl, at + 2 * wave + e);
            const uint64_t p = k8_uniform(a.c.codes + (size_t)ph[e] * head_bytes), ps = k8_uniform(a.c.scales + (size_t)ph[e] * head_scales);
            nk[e] = *reinterpret_cast<const __attribute__((address_space(1))) u32x4_k8*>(reinterpret_cast<gptr>(p) + kl * 16u);
            nv[e] = *reinterpret_cast<const __attribute__((address_space(1))) vlane*>(reinterpret_cast<gptr>(p) + (8 * HD + ln * (uint32_t)sizeof(vlane)));
            nks[e] = *reinterpret_cast<const __attribute__((address_space(1))) uint8_t*>(reinterpret_cast<gptr>(ps) + kl);
        }
        // lanes 0..15 and 16..31: the scales of V's sixteen positions of both pages
        const uint8_t* ps = a.c.scales + (size_t)(ln & 16 ? ph[1] : ph[0]) * head_scales + HD / 2 + (ln & 15);
        nvs = *ps;
    };
    auto put = [&](K4Stage<HD>& s) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (HD == 128 || lane < 32) *reinterpret_cast<u32x4_k8*>(s.k[2 * wave + e][lane]) = nk[e];
        *reinterpret_cast<uint16_t*>(&s.ks[lane][2 * wave]) = (uint16_t)(nks[0] | nks[1] << 8);
#pragma unroll
        for (int d = 0; d < DT; ++d) s.v[d][lane][wave] = __builtin_amdgcn_perm(nv[1][d / 2], nv[0][d / 2], d & 1 ? 0x07060302u : 0x05040100u);
        const unsigned long long odd = __ballot(nvs == 255u);
        const uint32_t b = nvs == 255u ? 0u : nvs;
        if (lane < 32) s.vs[2 * wave + (lane >> 4)][lane & 15] = __uint_as_float(b << 23);
        // (both halves of the wave have these bytes: one takes the largest, the other the least)
        const uint32_t m = k4_row_most(lane < 32 ? b : 255u - b);
        const auto of = [&](int at) { return (uint32_t)__builtin_amdgcn_readlane((int)m, at); };
        const uint32_t span = max(of(0), of(16)) | max(of(32), of(48)) << 16;
        if (lane == 0) {
            s.odd[wave] = (uint32_t)odd;
            s.span[wave] = span;
        }
    };

    // a lane's places in LDS
    uint32_t q16 = k4_lds_at(&sh.q[wave][0]) + 16 * lane;
    asm("" : "+v"(q16));
    uint32_t now = 0;
    if (steps) {
        fetch(0);
        put(sh.stage[group][0]);
    }
    if (group) __builtin_amdgcn_s_setprio(1);  // (the groups meet at every barrier, and would else want the same units at the same times)
    bool fresh = true;
    for (int st = 0; st < most; ++st) {
        const K4Stage<HD>& s = sh.stage[group][st & 1];
        now = map;
        __syncthreads();  // (also keeps the queries' reads in the loop: they are not held in registers)
        if (st + 1 < steps) fetch(st + 1);
        const int j0 = 16 * (pg0 + st * K4_STEP);
        // whether there is anything for this wave's tokens in these positions
        if (st < steps && j0 <= wp1 && !(a.window && j0 + 127 <= k8_hidden(a.window, wp0))) {
            const bool edge = now != 0xffu || j0 + 127 > wp0 || j0 + 128 > row.len || (a.window && j0 <= k8_hidden(a.window, wp1));
            constexpr uint32_t LO = offsetof(K4Query<HD>, lo), HI = offsetof(K4Query<HD>, hi), SC = offsetof(K4Query<HD>, scale);
            constexpr uint32_t SV = offsetof(K4Stage<HD>, v), SKS = offsetof(K4Stage<HD>, ks), SVS = offsetof(K4Stage<HD>, vs);
            uint32_t ln = lane;
            asm("" : "+v"(ln));
            const uint32_t base = k4_lds_at(&s), s16 = base + 16 * ln, sk = HD == 128 ? s16 : base + 16 * (ln & 31);
            const uint32_t odd = s.odd[0] | s.odd[1] | s.odd[2] | s.odd[3];
            float x[NT][32], l[NT];
            const auto mask = [&](int u) {
                if (CAP) k8_cap(reinterpret_cast<float(&)[1][32]>(x[u]), so);
                if (edge) {
                    const int pp = sh.pos[wave][u][lane & 15];
                    const int hi = min(pp, row.len - 1) - j0 - 4 * g, lo = (a.window ? k8_hidden(a.window, pp) : -1) - j0 - 4 * g;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int at = 16 * (i >> 2) + (i & 3);
                        x[u][i] = (now >> (i >> 2) & 1u) && at <= hi && at > lo ? x[u][i] : -__builtin_inff();
                    }
                }
                if (__any(odd != 0)) {  // a value of V that is not finite: the columns that see it, and no other, become NaN
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        x[u][i] = (s.odd[i >> 3] >> (4 * g) >> (16 * (i >> 2 & 1) + (i & 3)) & 1u) && x[u][i] != -__builtin_inff() ? __builtin_nanf("") : x[u][i];
                }
            };
            for (bool move = fresh;; move = true) {
                f32x4_k8 sc[NT][K4_STEP];
                const u32x2_k8 ks = k4_lds<u32x2_k8>(base + SKS + 8 * ln);
                uint32_t qs[NT];
                const uint32_t q8 = q16 - 8 * ln, q4 = q8 - 4 * ln;
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    qs[u] = k4_lds<uint32_t>(q4 + (uint32_t)(u * sizeof(K4Query<HD>)) + SC);
#pragma unroll
                    for (int e = 0; e < K4_STEP; ++e) sc[u][e] = f32x4_k8{0.f, 0.f, 0.f, 0.f};
                }
                u32x4_k8 kb[K4_STEP];
#pragma unroll
                for (int e = 0; e < K4_STEP; ++e) kb[e] = k4_lds<u32x4_k8>(sk + e * 8 * HD);
                // (a term's operands are requested before the products of the one before it)
                i32x6_k4 b[2][NT];
                const auto read = [&](int k) {
#pragma unroll
                    for (int u = 0; u < NT; ++u) {
                        const uint32_t at = (uint32_t)(u * sizeof(K4Query<HD>));
                        const u32x4_k8 lo = k4_lds<u32x4_k8>(q16 + at + LO + k * 1024);
                        const u32x2_k8 hi = k4_lds<u32x2_k8>(q8 + at + HI + k * 512);
                        b[k & 1][u] = i32x6_k4{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1]};
                    }
                    __builtin_amdgcn_sched_barrier(0);
                };
                const auto term = [&](auto K) {
#pragma unroll
                    for (int u = 0; u < NT; ++u) {
                        const i32x6_k4& o = b[K.value & 1][u];
                        sc[u][0] = k4_mfma<0, K.value>(kb[0], ks[0], o, qs[u], sc[u][0]);
                        sc[u][1] = k4_mfma<1, K.value>(kb[1], ks[0], o, qs[u], sc[u][1]);
                        sc[u][2] = k4_mfma<2, K.value>(kb[2], ks[0], o, qs[u], sc[u][2]);
                        sc[u][3] = k4_mfma<3, K.value>(kb[3], ks[0], o, qs[u], sc[u][3]);
                        sc[u][4] = k4_mfma<0, K.value>(kb[4], ks[1], o, qs[u], sc[u][4]);
                        sc[u][5] = k4_mfma<1, K.value>(kb[5], ks[1], o, qs[u], sc[u][5]);
                        sc[u][6] = k4_mfma<2, K.value>(kb[6], ks[1], o, qs[u], sc[u][6]);
                        sc[u][7] = k4_mfma<3, K.value>(kb[7], ks[1], o, qs[u], sc[u][7]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                };
                read(0);
                read(1);
                term(std::integral_constant<int, 0>{});
                if constexpr (K4_OPS<HD> == 3) read(2);
                term(std::integral_constant<int, 1>{});
                if constexpr (K4_OPS<HD> == 3) term(std::integral_constant<int, 2>{});
#pragma unroll
                for (int u = 0; u < NT; ++u) {
#pragma unroll
                    for (int e = 0; e < K4_STEP; ++e) asm volatile("" : "+v"(sc[u][e]));  // (here, not behind the branches that follow)
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[u][i] = sc[u][i >> 2][i & 3];
                }
                __builtin_amdgcn_sched_barrier(0);
                if (!REDO) break;
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    mask(u);
                    if (move) k4_move<HD>(k4_most(x[u]), so.f, acc[u]);
                    l[u] = k4_exp(x[u], so.f, acc[u].m);
                }
                if (move || !__any(l[0] > 0.5f || l[1] > 0.5f)) break;
            }
            fresh = false;
            int terms = 0;  // of the weights past two
            {
                uint32_t hi = 0, low = 0;  // (255 less the least)
#pragma unroll
                for (int w = 0; w < K8_WAVES; ++w) {
                    const uint32_t span = (uint32_t)__builtin_amdgcn_readfirstlane((int)s.span[w]);
                    hi = max(hi, span & 0xffffu);
                    low = max(low, span >> 16);
                }
                K4Apart d;
                d.lo = 255u - low;
                d.hi = hi;
                if (d.hi > d.lo + K4_NEAR) {
                    if (edge || d.lo <= K4_EMPTY) {  // of what some token of the wave sees
                        d = K4Apart{};
                        const int last = min(wp1, row.len - 1) - j0 - 4 * g, first = (a.window ? k8_hidden(a.window, wp0) : -1) - j0 - 4 * g;
#pragma unroll 1
                        for (int e = 0; e < K4_STEP; ++e)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                d.add(__float_as_uint(s.vs[e][4 * g + i]) >> 23, (now >> e & 1u) && 16 * e + i <= last && 16 * e + i > first);
                    }
                    terms = k4_wave_most(k4_terms(d.lo, d.hi));
                }
            }
            f32x16_k4 y[NT][2];
            i32x6_k4 p[NT][2];
            uint32_t ps[NT];
            const auto more = [&](int u) {
                k4_more<!CAP>(y[u][0], y[u][1], ps[u], terms, [&](const i32x6_k4& t, uint32_t b) {
                    asm volatile("" ::: "memory");  // (operands are read in each turn, not held in registers)
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        acc[u].o[d] = k4_mfma<0, 0>(k4_lds<u32x4_k8>(s16 + SV + d * 1024), 127u, t, b, acc[u].o[d]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                });
            };
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                if (REDO) {
                    acc[u].l += l[u];
                } else {
                    mask(u);
                    k4_probs<HD>(x[u], so.f, acc[u]);
                }
                float top = 0.0f;
#pragma unroll
                for (int e = 0; e < K4_STEP; ++e) {
                    const f32x4_k8 v = k4_lds<f32x4_k8>(base + SVS + 64 * e + 16 * g);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        y[u][i & 1][2 * e + (i >> 1)] = x[u][4 * e + i] * v[i];
                        top = fmaxf(top, y[u][i & 1][2 * e + (i >> 1)]);
                    }
                }
                ps[u] = k4_pair(y[u][0], y[u][1], top, p[u]);
                if (!LATE && terms) more(u);
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const u32x4_k8 A = k4_lds<u32x4_k8>(s16 + SV + d * 1024);
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    acc[u].o[d] = k4_mfma<0, 0>(A, 127u, p[u][0], ps[u], acc[u].o[d]);
                    acc[u].o[d] = k4_mfma<0, 1>(A, 127u, p[u][1], ps[u], acc[u].o[d]);
                }
            }
            if (LATE && terms) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int u = 0; u < NT; ++u) more(u);
            }
        }
        if (st + 1 < steps) put(sh.stage[group][(st + 1) & 1]);
    }
#pragma unroll
    for (int u = 0; u < NT; ++u) acc[u].l = k8_col_sum(acc[u].l);
    if constexpr (GROUPS == 2) {  // the second group's outputs join the first's, through the stages
        static_assert(K8_WAVES * NT * 64 * (DT * 4 + 2) * sizeof(float) <= sizeof(sh.stage), "a group's outputs fit the stages");
        f32x4_k8* other = reinterpret_cast<f32x4_k8*>(sh.stage) + wave * (NT * DT * 64) + lane;
        float* other_ml = reinterpret_cast<float*>(reinterpret_cast<f32x4_k8*>(sh.stage) + K8_WAVES * NT * DT * 64) + wave * (2 * NT * 64) + lane;
        __syncthreads();
        if (group) {
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                other_ml[2 * u * 64] = acc[u].m;
                other_ml[(2 * u + 1) * 64] = acc[u].l;
#pragma unroll
                for (int d = 0; d < DT; ++d) other[(u * DT + d) * 64] = acc[u].o[d];
            }
        }
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const float m1 = other_ml[2 * u * 64], M = fmaxf(acc[u].m, m1);
            const float f0 = k4_rescale(acc[u].m, M, so.f), f1 = k4_rescale(m1, M, so.f);
            acc[u].m = M;
            acc[u].l = acc[u].l * f0 + other_ml[(2 * u + 1) * 64] * f1;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[u].o[d] = acc[u].o[d] * f0 + other[(u * DT + d) * 64] * f1;
        }
    }
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const float L = acc[u].l;
        const float inv = L == 0.0f ? 0.0f : ieee_div(1.0f, L);
        const int rr = rr0 + 16 * u + c;
        if (rr >= live) continue;
        if (span.act > 1) {
            const size_t pr = ((size_t)(index * a.c.Hkv + kh) * nsplit + split) * ROWS + wave * (16 * NT) + 16 * u + c;
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4_k8*>(part + pr * HD + 16 * d + 4 * g) = acc[u].o[d];
            if (g == 0) {
                float* ml = part + (size_t)tiles * a.c.Hkv * nsplit * ROWS * HD + 2 * pr;
                ml[0] = acc[u].m;
                ml[1] = L;
            }
            continue;
        }
        uint16_t* out = k8_out(a, row, kh, rr) + 4 * g;
#pragma unroll
        for (int d = 0; d < DT; ++d)
            *reinterpret_cast<uint2*>(out + 16 * d) =
                make_uint2(k8_pack(acc[u].o[d][0] * inv, acc[u].o[d][1] * inv), k8_pack(acc[u].o[d][2] * inv, acc[u].o[d][3] * inv));
    }
}

// A call with longer rows: their blocks, then those of its rows of few query rows, in one launch.
template <int HD, int GROUPS, bool CAP>
__global__ __launch_bounds__(GROUPS* K8_THREADS) __attribute__((amdgpu_waves_per_eu(2))) void attn_kv4_mixed_kernel(
    Kv8AttnArgs a, K8Few few, int tiles, int csplit, float* cpart) {
    union Shared {
        K4ChunkShared<HD, GROUPS> chunk;
        K4FewShared<HD, GROUPS * K8_WAVES> few;
    };
    __shared__ __attribute__((aligned(16))) Shared sh;
    const int chunks = tiles * a.c.Hkv * csplit;
    if ((int)blockIdx.x < chunks)
        k4_chunk_block<HD, GROUPS, CAP>(a, 16, tiles, csplit, cpart, blockIdx.x, sh.chunk);
    else
        k4_few_block<HD, 1, GROUPS * K8_WAVES, CAP, false>(a, few, blockIdx.x - chunks, sh.few);
}

// Joins the splits of attn_kv4_mixed_kernel: blocks of its longer rows' tiles (csplit > 1), a wave per query row, then of the
// others.
template <int HD>
__global__ __launch_bounds__(K8_THREADS) void attn_kv4_mixed_join_kernel(Kv8AttnArgs a, K8Few few, int rowb, int tiles, int csplit,
                                                                        const float* cpart) {
    constexpr int ROWS = K4_CHUNK_ROWS, RB = ROWS / K8_WAVES;
    const int chunks = csplit > 1 ? tiles * a.c.Hkv * RB : 0;
    if ((int)blockIdx.x >= chunks) {
        k4_few_join<HD, 1, false>(a, few, blockIdx.x - chunks, rowb);
        return;
    }
    const int at = blockIdx.x / RB, kh = at % a.c.Hkv;
    const K8Tile tile = k8_tile<ROWS>(a, 16, at / a.c.Hkv);
    if (tile.r < 0) return;
    const K8Row row = k8_row(a, tile.r);
    const int i = blockIdx.x % RB * K8_WAVES + (threadIdx.x >> 6), rr = tile.t * ROWS + i;
    if (rr >= row.n * a.G) return;
    const int act = k8_span<ROWS, K4_STEP, K4_MIN_STAGES>(a, row, tile.t, csplit).act;
    if (act == 1) return;
    const size_t first = (size_t)at * csplit * ROWS + i;
    const float* ml = cpart + (size_t)tiles * a.c.Hkv * csplit * ROWS * HD;
    const float unit = k8_soft(a).f;
    k8_join<HD>(cpart + first * HD, (size_t)ROWS * HD, ml + 2 * first, 2 * ROWS, act, k8_out(a, row, kh, rr),
                [unit](float m, float M) { return k4_rescale(m, M, unit); });
}

// The launch.
struct K4Plan {
    int nt;                     // rows of few query rows: tiles of a block
    K8Few few;                  // and how they are split
    int64_t few_blocks;
    int64_t tiles;              // of K4_CHUNK_ROWS query rows, of the longer rows: at most (a row's last may be partly empty); 0: none
    int csplit;                 // splits of such a tile
    int groups;                 // of waves of a block in a call with longer rows
};
// Each choice with what was measured beside it (us; rows of one token with 32 query heads over 8 KV heads of 128, if not said otherwise):
// Rows of few query rows are split until there are two blocks of four waves a CU, or one of eight, which is what the registers let reside (four:
// 64 rows of 640 positions 19.8 instead of 13.7, 32 rows of 50 to 9000 45 instead of 42, 8 rows of 2000 the same; two of eight: 23 rows of four tokens
// behind 300 to 5000, 28 heads over 4, 27.2 instead of 20.0, 8 of six tokens behind 1000 to 4000 21.9 instead of 15.9).
constexpr int K4_BLOCKS_PER_CU = 2;
// Pages that a split takes at least: a step of every wave (half of that: one row of 512 8.5 instead of 6.1, for the join's launch, one of 16384 17.3
// instead of 12.5; twice: 8 rows of 2000 11.4 instead of 10.0),
constexpr int K4_MIN_PAGES = K4_STEP * K8_WAVES;
// and at most (256: 32 rows of 4096 to 16384 86.7 instead of 81.5),
constexpr int K4_MAX_PAGES = 1024;
// and beside longer rows, whose blocks take longer (64, 256, 512, 1024: 10 rows of 2000 to 15000 beside two chunks 247, 238, 238, 235 in all, three
// of 16000 beside a chunk of 40 59, 57, 57, 67, 20 rows of 40 to 4000 with a window of 1024 beside four 42.5, 38.9, 38.8, 38.9).
constexpr int K4_MIXED_PAGES = 512;
constexpr int K4_MAX_SPLITS = 64;
// From splits of so many pages on, the blocks find from all lengths how few pages a split may take (never: 32 rows of 4096 to 16384 88.3 instead of 81.5, of
// 50 to 9000 48.6 instead of 41.6; from 16 pages on: 8 rows of 2000 12.6 instead of 10.0, for the lengths that every block then reads).
constexpr int K4_EVEN_PAGES = 64;
// Longer rows: tiles are split while they leave CUs without a block (two blocks a CU: a prompt of 1000 46 instead of 26, a chunk of 300 behind 8000 77
// instead of 66, as the splits' outputs are written and joined; a chunk of 40 beside three rows of 16000 46 instead of 57). Splits of 2 and of 8 steps at least
// were as fast as of 4.
constexpr int K4_CHUNK_BLOCKS_PER_CU = 1;
// A block has two groups of waves up to so many blocks a CU (always: four chunks of 2048 588 instead of 522; never: a prompt of 2001 59 instead
// of 51, the mixed batch of 20 tokens and 4 chunks 48 instead of 39).
constexpr int K4_GROUP_BLOCKS_PER_CU = 2;
// pages that a group of `tokens` neighbouring tokens of a row sees at most, by the host's bounds
int64_t pages_seen(const Kv8AttnArgs& a, int64_t tokens) {
    int64_t len = a.max_len;
    if (a.window) len = std::min<int64_t>(len, (int64_t)a.window + tokens + 15);
    return std::max<int64_t>(1, (len + 15) / 16);
}
K4Plan plan_of(const Kv8AttnArgs& a) {
    K4Plan p;
    const int64_t rows = (int64_t)a.max_new * a.G;
    p.tiles = rows <= 32 ? 0 : (int64_t)a.T * a.G / K4_CHUNK_ROWS + std::min(a.B, a.T);
    p.nt = rows <= 16 || p.tiles ? 1 : 2;
    const int64_t pages = pages_seen(a, std::min(a.max_new, 16 * p.nt / a.G));
    const int64_t blocks = (int64_t)a.B * a.c.Hkv;
    const int reside = K4_BLOCKS_PER_CU * a.n_cu / p.nt;
    const int64_t want = std::max<int64_t>(1, (reside + blocks / 2) / blocks);
    int64_t sp = std::min<int64_t>(K4_MAX_PAGES, std::max<int64_t>(K4_MIN_PAGES, (pages + want - 1) / want));
    if (p.tiles) sp = std::min<int64_t>(K4_MIXED_PAGES, pages);
    sp = std::max(sp, (pages + K4_MAX_SPLITS - 1) / K4_MAX_SPLITS);
    const int nsplit = (int)((pages + sp - 1) / sp);
    const int units = reside / a.c.Hkv;
    p.few = K8Few{(int)sp, nsplit, nsplit, 0};
    p.few_blocks = blocks * nsplit;
    if (!p.tiles && nsplit > 1 && sp >= K4_EVEN_PAGES && a.B > 1 && a.B <= 64 && a.B < units && (int64_t)a.B * a.maxp <= 1 << 30) {
        p.few.most = std::min(2 * nsplit, K4_MAX_SPLITS);
        p.few.units = units;
        p.few_blocks = std::max<int64_t>(p.few_blocks, (int64_t)units * a.c.Hkv);
    }
    p.csplit = p.groups = 1;
    if (p.tiles) {
        const int64_t stages = (pages_seen(a, std::min(a.max_new, K4_CHUNK_ROWS / a.G + 1)) + K4_STEP - 1) / K4_STEP;
        const int64_t most = std::min<int64_t>(K4_MAX_SPLITS, std::max<int64_t>(1, stages / K4_MIN_STAGES));
        p.csplit = (int)std::min<int64_t>(most, std::max<int64_t>(1, K4_CHUNK_BLOCKS_PER_CU * a.n_cu / (p.tiles * a.c.Hkv)));
        p.groups = p.tiles * a.c.Hkv * p.csplit <= K4_GROUP_BLOCKS_PER_CU * a.n_cu ? 2 : 1;
    }
    return p;
}

size_t few_floats(const Kv8AttnArgs& a, const K4Plan& p) {
    return p.few.nsplit == 1 ? 0 : (size_t)a.B * a.c.Hkv * p.few.most * (16 * p.nt) * (a.c.hd + 2);
}

template <int HD, int NT, bool EVEN>
void launch_few(const Kv8AttnArgs& a, const K4Plan& p, int rowb, int64_t joins, hipStream_t s) {
    constexpr int WAVES = NT * K8_WAVES;
    auto f = a.cap > 0.0f ? attn_kv4_few_kernel<HD, NT, WAVES, true, EVEN> : attn_kv4_few_kernel<HD, NT, WAVES, false, EVEN>;
    hipLaunchKernelGGL(f, dim3((unsigned)p.few_blocks), dim3(64 * WAVES), 0, s, a, p.few);
    if (joins)
        hipLaunchKernelGGL((attn_kv4_join_kernel<HD, NT, EVEN>), dim3((unsigned)joins), dim3(K8_THREADS), 0, s, a, p.few, rowb);
}
template <int HD>
void launch(const Kv8AttnArgs& a, const K4Plan& p, hipStream_t s) {
    const int rowb = (int)(std::min<int64_t>((int64_t)a.max_new * a.G, 16 * p.nt) + K8_WAVES - 1) / K8_WAVES;
    const int64_t few_joins = p.few.nsplit > 1 ? (int64_t)a.B * a.c.Hkv * rowb : 0;
    if (p.tiles == 0) {
        auto f = p.nt == 2 ? (p.few.units ? launch_few<HD, 2, true> : launch_few<HD, 2, false>)
                           : (p.few.units ? launch_few<HD, 1, true> : launch_few<HD, 1, false>);
        f(a, p, rowb, few_joins, s);
        return;
    }
    float* cpart = a.part + few_floats(a, p);
    const dim3 grid((unsigned)(p.tiles * a.c.Hkv * p.csplit + p.few_blocks));
    auto f = p.groups == 2 ? (a.cap > 0.0f ? attn_kv4_mixed_kernel<HD, 2, true> : attn_kv4_mixed_kernel<HD, 2, false>)
                           : (a.cap > 0.0f ? attn_kv4_mixed_kernel<HD, 1, true> : attn_kv4_mixed_kernel<HD, 1, false>);
    hipLaunchKernelGGL(f, grid, dim3(p.groups * K8_THREADS), 0, s, a, p.few, (int)p.tiles, p.csplit, cpart);
    const int64_t joins = few_joins + (p.csplit > 1 ? p.tiles * a.c.Hkv * (K4_CHUNK_ROWS / K8_WAVES) : 0);
    if (joins)
        hipLaunchKernelGGL(attn_kv4_mixed_join_kernel<HD>, dim3((unsigned)joins), dim3(K8_THREADS), 0, s, a, p.few, rowb,
                           (int)p.tiles, p.csplit, cpart);
}

}  // namespace

size_t kv4_attention_ws_bytes(const Kv8AttnArgs& a) {
    const K4Plan p = plan_of(a);
    const size_t chunk = p.csplit == 1 ? 0 : (size_t)p.tiles * a.c.Hkv * p.csplit * K4_CHUNK_ROWS * (a.c.hd + 2);
    return (few_floats(a, p) + chunk) * sizeof(float);
}

bool kv4_attention_fits(const Kv8AttnArgs& a) {
    const K4Plan p = plan_of(a);
    constexpr int64_t most = 1 << 22;  // blocks of a launch
    return (int64_t)a.T * a.G <= (1 << 29) && p.tiles * a.c.Hkv * p.csplit + p.few_blocks <= most &&
           (int64_t)a.B * a.c.Hkv * 8 + p.tiles * a.c.Hkv * (p.csplit > 1 ? K4_CHUNK_ROWS / K8_WAVES : 0) <= 2 * most;
}

hipError_t launch_kv4_attention(const Kv8AttnArgs& a, hipStream_t s) {
    const K4Plan p = plan_of(a);
    if (a.c.hd == 128)
        launch<128>(a, p, s);
    else
        launch<64>(a, p, s);
    return hipGetLastError();
}

}  // namespace mg
