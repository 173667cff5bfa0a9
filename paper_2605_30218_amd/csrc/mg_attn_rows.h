// mg_attn_rows.h -- what the attention kernels of the 8-bit and the 4-bit paged cache share: the rows of a call and what their
// tokens see, splits of rows and tiles over positions, capped scores, and the join of splits.
#pragma once
#include "mg_device.h"
#include "mg_kernels.h"

namespace mg {

typedef __bf16 bf16x2_k8 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_k8 __attribute__((ext_vector_type(8)));
typedef float f32x4_k8 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_k8 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_k8 __attribute__((ext_vector_type(4)));

constexpr int K8_WAVES = 4;
constexpr int K8_THREADS = 64 * K8_WAVES;
constexpr int K8_IDS = 64;  // page ids a wave holds at a time, one a lane

// bf16 pair nearest to two floats, ties to even
__device__ __forceinline__ uint32_t k8_pack(float lo, float hi) {
    bf16x2_k8 v;
    v.x = (__bf16)lo;
    v.y = (__bf16)hi;
    return __builtin_bit_cast(uint32_t, v);
}
// 16 bytes at a wave-uniform address and a lane's own offset; the address stays in scalar registers
__device__ __forceinline__ uint64_t k8_uniform(const uint8_t* p) {
    const uint64_t u = reinterpret_cast<uint64_t>(p);
    uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
    asm("" : "+s"(lo), "+s"(hi));
    return lo | (uint64_t)hi << 32;
}
__device__ __forceinline__ u32x4_k8 k8_load(uint64_t p, uint32_t off) {
    typedef const __attribute__((address_space(1))) char* gptr;
    return *reinterpret_cast<const __attribute__((address_space(1))) u32x4_k8*>(reinterpret_cast<gptr>(p) + off);
}
// a lane's row c, all four lanes c, c + 16, c + 32, c + 48
__device__ __forceinline__ float k8_col_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float k8_col_sum(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// What a row's tokens see: token i stands at p0 + i and sees the mapped positions of [0, len) that are
// <= p0 + i and, with a window, > p0 + i - window.  A token stands anywhere below 2^31 (past the page table too) and a
// window is any, so p - window is only taken where it is at least -1.
struct K8Row {
    int t0, n;      // its tokens of q
    int len, p0;    // positions in reach of the page table; position of its first token
    int pga, pgb;   // pages that any of its tokens sees: [pga, pgb)
};
// the last position that the window hides from a token at p, or -1
__device__ __forceinline__ int k8_hidden(int window, int p) { return max(p, window - 1) - window; }
__device__ __forceinline__ int k8_token(const Kv8AttnArgs& a, int t) { return min(max(t, 0), a.T); }
__device__ __forceinline__ K8Row k8_row(const Kv8AttnArgs& a, int r) {
    K8Row x;
    x.t0 = a.cu_new ? k8_token(a, a.cu_new[r]) : r;
    x.n = (a.cu_new ? k8_token(a, a.cu_new[r + 1]) : r + 1) - x.t0;
    const int len = max(a.lens[r], 0);
    x.len = min(len, 16 * a.maxp);
    x.p0 = len - x.n;
    x.pga = a.window ? min(k8_hidden(a.window, x.p0) + 1, x.len) / 16 : 0;
    x.pgb = (x.len + 15) / 16;
    return x;
}
constexpr int K8_MIN_PAGES = 8;  // pages a split takes at least: a step of every wave
// How rows of few query rows are split: pages of a split, splits of a row at most.  units > 0 (at most 64 rows): a split takes
// fewer pages, down to sp / 2, as long as the splits of all rows together are at most `units`; most: the splits of a row then.
struct K8Few {
    int sp, nsplit, most, units;
};
// splits of npg pages among at most nsplit blocks of about sp pages (an even number each)
__device__ __forceinline__ int k8_active(int npg, int sp, int nsplit) {
    return min(nsplit, max(1, (npg + sp - 1) / sp));
}
// Lane r: row r, its splits (0 where it has no tokens or more than LIMIT query rows), and those of the rows up to it.  All
// lanes find the same pages of a split.
struct K8Lanes {
    K8Row row;
    int act, sum;
};
template <int LIMIT>
__device__ __forceinline__ K8Lanes k8_lanes(const Kv8AttnArgs& a, const K8Few& p) {
    const int lane = threadIdx.x & 63;
    K8Lanes x;
    x.row = k8_row(a, min(lane, a.B - 1));
    const bool live = lane < a.B && x.row.n > 0 && x.row.n * a.G <= LIMIT;
    const int npg = live ? max(x.row.pgb - x.row.pga, 0) : 0;
    int total = npg;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) total += __shfl_xor(total, o, 64);
    const int rows = __popcll(__ballot(live));
    auto split = [&](int sp) {
        x.act = live ? k8_active(npg, sp, sp == p.sp ? p.nsplit : p.most) : 0;
        x.sum = x.act;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(x.sum, o, 64);
            if (lane >= o) x.sum += v;
        }
        return __builtin_amdgcn_readlane(x.sum, 63);
    };
    // a row's last split is half empty on average, wholly at worst: rows / 2 splits more than total / sp, or rows
    auto pages = [&](int splits) {
        return min(p.sp, max(max(p.sp / 2, K8_MIN_PAGES), (total + splits - 1) / max(splits, 1)));
    };
    const int sp = pages(p.units - rows / 2);
    if (split(sp) > p.units && sp < p.sp) split(pages(p.units - rows));
    return x;
}
__device__ __forceinline__ K8Row k8_of_lane(const K8Row& x, int at) {
    return K8Row{__builtin_amdgcn_readlane(x.t0, at), __builtin_amdgcn_readlane(x.n, at), __builtin_amdgcn_readlane(x.len, at),
                 __builtin_amdgcn_readlane(x.p0, at), __builtin_amdgcn_readlane(x.pga, at), __builtin_amdgcn_readlane(x.pgb, at)};
}

// what the kernels derive from the scale and the cap: the exponent is x * f with x a product q . k or what k8_cap makes of it
struct K8Soft {
    float f, zin, most;  // most: of |q . k| up to which z is at most 1/2
};
__device__ __forceinline__ K8Soft k8_soft(const Kv8AttnArgs& a) {
    constexpr float log2e = 1.4426950408889634f;
    const float zin = a.scale * a.inv_cap;
    return K8Soft{(a.cap > 0.0f ? a.cap : a.scale) * log2e, zin, 0.5f * ieee_div(1.0f, zin)};
}

// Capped scores: a step's products q . k become tanh(z), z = scale * q . k / cap.  Up to 1/2 by a polynomial that is off by 2^-25 of
// tanh (fitted to tanh(z) / z - 1 over z^2, relative errors least), without a transcendental instruction; a step that
// has larger ones takes 1 - 2 / (1 + e^2z) for those, off by some 2^-23.  So a score keeps its relative accuracy whatever
// the cap.
template <int NT, int N>
__device__ __forceinline__ void k8_cap(float (&x)[NT][N], const K8Soft& so) {
    float top = 0.0f;
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, __builtin_fabsf(x[u][i]));
    const bool large = __any(!(top <= so.most));
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float z = x[u][i] * so.zin, zz = z * z;
            float t = __builtin_fmaf(z * zz, __builtin_fmaf(zz, __builtin_fmaf(zz, __builtin_fmaf(zz, 0.01724149f, -0.05304549f), 0.13325879f), -0.33333144f), z);
            if (large) {
                const float e = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(2.8853900817779268f * z));
                t = __builtin_fabsf(z) <= 0.5f ? t : e;
            }
            x[u][i] = t;
        }
}

// The factor of what was summed under an exponents' reference m (log2 units) where the reference is M.
struct K8Weight {
    __device__ __forceinline__ float operator()(float m, float M) const { return __builtin_amdgcn_exp2f(m - M); }
};
// One query row's splits joined in their order by a wave: outputs at po + s * so, reference and sum of split s in lane s's
// ml (act <= 64); weight: as K8Weight.
template <int HD, class Weight = K8Weight>
__device__ __forceinline__ void k8_join(const float* po, size_t so, const float* pml, size_t sml, int act, uint16_t* out, Weight weight = Weight{}) {
    constexpr int PL = HD / 64;  // consecutive features of a lane
    constexpr int AHEAD = 8;     // splits whose outputs are requested together, the first before their weights are known
    const int lane = threadIdx.x & 63;
    using vec = float __attribute__((ext_vector_type(PL)));
    vec v[AHEAD];
    const float2 ml = *reinterpret_cast<const float2*>(pml + (size_t)min(lane, act - 1) * sml);
    po += PL * lane;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) v[k] = *reinterpret_cast<const vec*>(po + (size_t)min(k, act - 1) * so);
    const float M = wave_max(ml.x);
    const float f = lane < act ? weight(ml.x, M) : 0.0f;
    const float L = wave_sum_fast(lane < act ? f * ml.y : 0.0f);
    const float inv = L == 0.0f ? 0.0f : ieee_div(1.0f, L);
    float O[PL];
#pragma unroll
    for (int e = 0; e < PL; ++e) O[e] = 0.0f;
    for (int s = 0; s < act; s += AHEAD) {
        if (s) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) v[k] = *reinterpret_cast<const vec*>(po + (size_t)min(s + k, act - 1) * so);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (s + k >= act) break;
            const float w = __shfl(f, s + k, 64);
#pragma unroll
            for (int e = 0; e < PL; ++e) O[e] += w * v[k][e];
        }
    }
    out += PL * lane;
    if constexpr (PL == 2)
        *reinterpret_cast<uint32_t*>(out) = k8_pack(O[0] * inv, O[1] * inv);
    else
        out[0] = (uint16_t)f2bf(O[0] * inv);
}
__device__ __forceinline__ uint16_t* k8_out(const Kv8AttnArgs& a, const K8Row& row, int kh, int rr) {
    return a.out + (int64_t)(row.t0 + rr / a.G) * a.out_stride + (size_t)(kh * a.G + rr % a.G) * a.c.hd;
}

// Tile `index` of the rows of more than `few` query rows, their tiles of ROWS query rows counted row by row: the row, and the
// tile in it from its end (the last tokens see the most); r < 0 behind the last.  Tile counts are summed by
// the wave, 64 rows at a time.
struct K8Tile {
    int r, t;
};
template <int ROWS>
__device__ __forceinline__ K8Tile k8_tile(const Kv8AttnArgs& a, int few, int index) {
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        int k = 0;
        if (b0 + lane < a.B) {
            const int rows = (k8_token(a, a.cu_new[b0 + lane + 1]) - k8_token(a, a.cu_new[b0 + lane])) * a.G;
            k = rows > few ? (rows + ROWS - 1) / ROWS : 0;
        }
        int sum = k;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(sum, o, 64);
            if (lane >= o) sum += v;
        }
        const unsigned long long past = __ballot(sum > index);
        if (past) {
            const int at = __builtin_amdgcn_readfirstlane(__ffsll(past) - 1);
            return K8Tile{b0 + at, __builtin_amdgcn_readlane(sum, at) - 1 - index};
        }
        index -= __builtin_amdgcn_readlane(sum, 63);
    }
    return K8Tile{-1, 0};
}
// The pages that tile t's tokens see, the stages of STAGE pages they make and the splits that share these, at least
// MIN_STAGES each.
struct K8Span {
    int pg0, pg1, stages, act;
};
template <int ROWS, int STAGE, int MIN_STAGES>
__device__ __forceinline__ K8Span k8_span(const Kv8AttnArgs& a, const K8Row& row, int t, int nsplit) {
    const int p0 = row.p0 + t * ROWS / a.G, p1 = row.p0 + (min((t + 1) * ROWS, row.n * a.G) - 1) / a.G;
    K8Span x;
    x.pg0 = a.window ? min(k8_hidden(a.window, p0) + 1, row.len) / 16 : 0;
    x.pg1 = max(0, min(p1 + 1, row.len) + 15) / 16;
    x.stages = max(0, (x.pg1 - x.pg0 + STAGE - 1) / STAGE);
    x.act = max(1, min(nsplit, x.stages / MIN_STAGES));
    return x;
}

}  // namespace mg
