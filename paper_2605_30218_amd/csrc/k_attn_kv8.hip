// k_attn_kv8.hip -- attention of a batch's new tokens over the 8-bit paged K/V cache.
//
// out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m) in one pass over the positions, with a running reference m.  Two
// kinds of blocks, both S^T = K Q^T and O^T = V^T P^T on the matrix cores with K and V as A operands straight in the
// order in which the cache stores a page: "few" blocks for rows of at most 16 or 32 query rows (single tokens,
// drafts), bound by the K/V stream, split over positions and joined where rows are few; "chunk" blocks for longer rows,
// bound by the matrix cores and the vector units together.  A call without longer rows launches few blocks, one
// with them both kinds in one grid.
// Measured, hd 128 (us of a call in a captured graph): 64 rows of 512..768, 32 heads over 8: 19.0 (85 MB, 4.5 TB/s);
// 128 rows of 127..2047, 40 over 8: 60.4 (4.8 TB/s); 32 rows of 4095..16383: 121 (5.5 TB/s; a streaming read
// 6.2); 23 rows of four tokens, 28 over 4: 27.0; one prompt of 2001, 28 over 4: 50 (580 TFLOP/s); 4 chunks of 2048 behind
// up to 6144: 580 (948 TFLOP/s; a library's product of 8192^3: 1390), once the card is in step: the first 40 runs after an
// idle second take 730 down to 600.
#include <algorithm>

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

// four e4m3 codes times 2^(b - 127) (the float `scale`) as two bf16 pairs, exact
__device__ __forceinline__ uint2 k8_bf16x4(uint32_t w, float scale) {
    const bf16x2_k8 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    const bf16x2_k8 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
    return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}
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
// Codes that are not finite in bf16: NaN, and those that stand for 2^128 or more, which only pages of scale bytes above 246
// have (a code of exponent e stands for 2^(e - 7 + b - 127) and up, so e >= 262 - b).  k8_odd_add: what takes the
// least such code under scale 2^(b - 127) (the float `scale`) to 0x80, in every byte; k8_odd_bytes: the high bit of each.
__device__ __forceinline__ uint32_t k8_odd_add(float scale) {
    const uint32_t b = __float_as_uint(scale) >> 23;
    return 0x01010101u * (b < 247u ? 1u : 8u * (b - 246u));
}
__device__ __forceinline__ uint32_t k8_odd_bytes(uint32_t w, uint32_t add) { return ((w & 0x7f7f7f7fu) + add) & 0x80808080u; }

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

// ---- one step: 32 positions (two pages) against NT tiles of 16 query rows
// S^T[pos][c] = K[pos][:] . Q[c][:]: K is the A operand, straight from a page (the cache stores a head's
// page in the order in which a wave's 16-byte reads give the operand registers), and column c of a
// tile one query row, in lanes c, c + 16, c + 32, c + 48.
// O^T[d][c] += V^T[d][pos] P^T[pos][c]: V is the A operand, likewise; the scores' registers, positions
// 4 g .. 4 g + 3 of both pages in lane group g, are the B operand as they are.
// So a row's maximum takes two exchanges between lanes, and its rescaling is a lane's own.  Codes become bf16 with
// their page's scale in one instruction a pair, exactly.
template <int HD, int NT>
struct K8Acc {
    float m[NT], l[NT];          // reference of the exponents (log2 units); sum over the lane's positions
    f32x4_k8 o[NT][HD / 16];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            // below every finite score, and finite: exp2(masked - m) is 0 where nothing was seen yet
            m[u] = -3.0e38f;
            l[u] = 0.0f;
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) o[u][d] = f32x4_k8{0.f, 0.f, 0.f, 0.f};
        }
    }
};
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
template <int NT>
__device__ __forceinline__ void k8_cap(float (&x)[NT][8], const K8Soft& so) {
    float top = 0.0f;
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, __builtin_fabsf(x[u][i]));
    const bool large = __any(!(top <= so.most));
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float z = x[u][i] * so.zin, zz = z * z;
            float t = __builtin_fmaf(z * zz, __builtin_fmaf(zz, __builtin_fmaf(zz, __builtin_fmaf(zz, 0.01724149f, -0.05304549f), 0.13325879f), -0.33333144f), z);
            if (large) {
                const float e = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(2.8853900817779268f * z));
                t = __builtin_fabsf(z) <= 0.5f ? t : e;
            }
            x[u][i] = t;
        }
}

// scores: x[u][4 e + i] of position 16 e + 4 g + i of the step and column c of tile u
template <int HD, int NT, bool CAP>
__device__ __forceinline__ void k8_scores(const uint4 (&kb)[2][HD / 64], const float (&ksc)[2],
                                          const uint4 (&qa)[NT][HD / 32], const K8Soft& so, float (&x)[NT][8]) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        f32x4_k8 acc[NT];
#pragma unroll
        for (int u = 0; u < NT; ++u) acc[u] = f32x4_k8{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < HD / 64; ++h)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const uint2 lo = k8_bf16x4(st ? kb[e][h].z : kb[e][h].x, ksc[e]);
                const uint2 hi = k8_bf16x4(st ? kb[e][h].w : kb[e][h].y, ksc[e]);
                const bf16x8_k8 A = __builtin_bit_cast(bf16x8_k8, make_uint4(lo.x, lo.y, hi.x, hi.y));
#pragma unroll
                for (int u = 0; u < NT; ++u)
                    acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, __builtin_bit_cast(bf16x8_k8, qa[u][2 * h + st]), acc[u], 0, 0, 0);
            }
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[u][4 * e + i] = acc[u][i];
    }
    if (CAP) k8_cap<NT>(x, so);
}

// Whether the token at position p sees the step's position i of this lane: j0 the step's first position,
// mapped bit e whether page e is one of the cache's.
__device__ __forceinline__ bool k8_sees(const K8Row& row, int window, int j0, int mapped, int g, int i, int p) {
    const int j = j0 + 16 * (i >> 2) + 4 * g + (i & 3);
    return ((mapped >> (i >> 2)) & 1) && j <= p && j < row.len && (!window || j > k8_hidden(window, p));
}

// The online softmax of a step.  The reference m moves only when a row's probabilities of the step would sum to more than
// K8_MOVE on a lane: their bits are relative, and the exchanges between lanes and the rescaling of the
// output are rare (the sums, which are needed anyway, tell; a reference far too low makes infinities, which are
// more).  TERMS bf16 values stand for a probability: their sum is 2^-8 (1) or 2^-16 (2) of itself off.  Two where
// the K/V stream bounds a block, one in chunks, where the second product takes 4 chunks of 2048 from 580 to 727 us, a prompt of
// 2001 from 51 to 60 and the outputs' error, relative to the result, from 0.0021 to 0.0016, that of their own rounding to bf16.
constexpr float K8_MOVE = 4096.0f;
template <int HD, int NT, int TERMS>
__device__ __forceinline__ void k8_softmax(const float (&x)[NT][8], float f, K8Acc<HD, NT>& acc, bf16x8_k8 (&p)[NT][TERMS]) {
    float y[NT][8], t[NT];
    bool move = false;
    auto probs = [&](int u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[u][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][i], f, -acc.m[u]));
        t[u] = ((y[u][0] + y[u][1]) + (y[u][2] + y[u][3])) + ((y[u][4] + y[u][5]) + (y[u][6] + y[u][7]));
    };
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        probs(u);
        move |= t[u] > K8_MOVE;
    }
    if (__any(move)) {
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const float mx = fmaxf(fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3])),
                                   fmaxf(fmaxf(x[u][4], x[u][5]), fmaxf(x[u][6], x[u][7])));
            const float mn = fmaxf(acc.m[u], k8_col_max(mx) * f);
            const float al = __builtin_amdgcn_exp2f(acc.m[u] - mn);
            acc.m[u] = mn;
            acc.l[u] *= al;
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) acc.o[u][d] *= al;
            probs(u);
        }
    }
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        acc.l[u] += t[u];
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = k8_pack(y[u][2 * i], y[u][2 * i + 1]);
        p[u][0] = __builtin_bit_cast(bf16x8_k8, make_uint4(w[0], w[1], w[2], w[3]));
        if constexpr (TERMS == 2) {
            uint32_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = k8_pack(y[u][2 * i] - bf_lo(w[i]), y[u][2 * i + 1] - bf_hi(w[i]));
            p[u][1] = __builtin_bit_cast(bf16x8_k8, make_uint4(v[0], v[1], v[2], v[3]));
        }
    }
}

// A value of V that is not finite, under a probability of zero: in a step whose columns do not all see all positions it
// must reach the columns that see it and no other.  Takes these codes out of vb and puts a NaN into the outputs
// that see one, found by a product of the codes' and the columns' indicators.
template <int HD, int NT>
__device__ __forceinline__ void k8_mend_odd(uint4 (&vb)[2][HD / 64], const float (&vsc)[2], K8Acc<HD, NT>& acc, const K8Row& row,
                                            int window, int j0, int mapped, int g, const int (&pc)[NT]) {
    const uint32_t add[2] = {k8_odd_add(vsc[0]), k8_odd_add(vsc[1])};
    uint32_t any = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int h = 0; h < HD / 64; ++h)
            any |= k8_odd_bytes(vb[e][h].x, add[e]) | k8_odd_bytes(vb[e][h].y, add[e]) | k8_odd_bytes(vb[e][h].z, add[e]) |
                   k8_odd_bytes(vb[e][h].w, add[e]);
    if (!__any(any != 0)) return;
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        uint32_t sw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            sw[i] = (k8_sees(row, window, j0, mapped, g, 2 * i, pc[u]) ? 0x3f80u : 0u) |
                    (k8_sees(row, window, j0, mapped, g, 2 * i + 1, pc[u]) ? 0x3f800000u : 0u);
        const bf16x8_k8 S = __builtin_bit_cast(bf16x8_k8, make_uint4(sw[0], sw[1], sw[2], sw[3]));
#pragma unroll
        for (int h = 0; h < HD / 64; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t f[4];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t nb = k8_odd_bytes(q == 0 ? vb[e][h].x : q == 1 ? vb[e][h].y : q == 2 ? vb[e][h].z : vb[e][h].w, add[e]);
                    f[2 * e] = ((nb >> 7) & 1u) * 0x3f80u | ((nb >> 15) & 1u) * 0x3f800000u;
                    f[2 * e + 1] = ((nb >> 23) & 1u) * 0x3f80u | (nb >> 31) * 0x3f800000u;
                }
                f32x4_k8 hit = f32x4_k8{0.f, 0.f, 0.f, 0.f};
                hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_k8, make_uint4(f[0], f[1], f[2], f[3])), S, hit, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc.o[u][4 * h + q][i] = hit[i] > 0.0f ? __builtin_nanf("") : acc.o[u][4 * h + q][i];
            }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int h = 0; h < HD / 64; ++h) {
            vb[e][h].x &= ~((k8_odd_bytes(vb[e][h].x, add[e]) >> 7) * 0xffu);
            vb[e][h].y &= ~((k8_odd_bytes(vb[e][h].y, add[e]) >> 7) * 0xffu);
            vb[e][h].z &= ~((k8_odd_bytes(vb[e][h].z, add[e]) >> 7) * 0xffu);
            vb[e][h].w &= ~((k8_odd_bytes(vb[e][h].w, add[e]) >> 7) * 0xffu);
        }
}

template <int HD, int NT, int TERMS>
__device__ __forceinline__ void k8_pv(const uint4 (&vb)[2][HD / 64], const float (&vsc)[2], const bf16x8_k8 (&p)[NT][TERMS],
                                      K8Acc<HD, NT>& acc) {
#pragma unroll
    for (int h = 0; h < HD / 64; ++h)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t w0 = q == 0 ? vb[0][h].x : q == 1 ? vb[0][h].y : q == 2 ? vb[0][h].z : vb[0][h].w;
            const uint32_t w1 = q == 0 ? vb[1][h].x : q == 1 ? vb[1][h].y : q == 2 ? vb[1][h].z : vb[1][h].w;
            const uint2 lo = k8_bf16x4(w0, vsc[0]), hi = k8_bf16x4(w1, vsc[1]);
            const bf16x8_k8 A = __builtin_bit_cast(bf16x8_k8, make_uint4(lo.x, lo.y, hi.x, hi.y));
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int t = 0; t < TERMS; ++t)
                    acc.o[u][4 * h + q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, p[u][t], acc.o[u][4 * h + q], 0, 0, 0);
        }
}

// query rows rr0 + 16 u + c of a row's KV head (row rr: token rr / G, head rr % G of the group) as B operands, and
// the positions of their tokens; columns past the row's last repeat its first
template <int HD, int NT>
__device__ __forceinline__ void k8_query(const Kv8AttnArgs& a, const K8Row& row, int kh, int rr0, int c, int g,
                                         uint4 (&qa)[NT][HD / 32], int (&pc)[NT]) {
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        int rr = rr0 + 16 * u + c;
        rr = rr < row.n * a.G ? rr : 0;
        const uint16_t* qp = a.q + (int64_t)(row.t0 + rr / a.G) * a.q_stride + (size_t)(kh * a.G + rr % a.G) * HD;
        pc[u] = row.p0 + rr / a.G;
#pragma unroll
        for (int h = 0; h < HD / 64; ++h) {
            // operand slot (g, st) holds features 64 h + 16 g + 8 st ..
            qa[u][2 * h] = *reinterpret_cast<const uint4*>(qp + 64 * h + 16 * g);
            qa[u][2 * h + 1] = *reinterpret_cast<const uint4*>(qp + 64 * h + 16 * g + 8);
        }
    }
}

// Rows of few query rows (tokens times query heads of a KV head <= 16 NT): one block per (row, KV head,
// split of the row's pages), a wave taking every WAVES-th step of its pages.  The K/V stream
// bounds it, so the matrix cores have the time for two terms of a probability.  K's registers are loaded again as
// soon as the scores are there, V's after its product, so that a wave has a step in flight at any time.  Pages are read once:
// loads that leave no trace in the caches (32 rows of 4096..16384: 138 -> 122 us, 128 ragged rows 67.7 -> 60.4; only
// what the memory-side cache still holds from the call before is slower, 64 MB of 23 rows 26.0 -> 27.5).
template <int HD, int NT, int WAVES>
struct K8FewShared {
    float o[WAVES][16 * NT][HD + 4];  // (padded rows)
    float m[WAVES][16 * NT], l[WAVES][16 * NT];
};
template <int HD, int NT, int WAVES, bool CAP, bool EVEN>
__device__ __forceinline__ void k8_few_block(const Kv8AttnArgs& a, const K8Few& few, int block, K8FewShared<HD, NT, WAVES>& sh) {
    constexpr int H = HD / 64;        // 1 KiB runs of a page of K or V
    constexpr int DT = HD / 16;       // output tiles
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
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
    const int per = ((npg + act - 1) / act + 1) & ~1;
    const int pg0 = row.pga + split * per, pg1 = split == act - 1 ? row.pgb : min(row.pgb, pg0 + per);

    uint4 qa[NT][2 * H];
    int pc[NT];
    k8_query<HD, NT>(a, row, kh, 0, c, g, qa, pc);
    const K8Soft so = k8_soft(a);
    K8Acc<HD, NT> acc;
    acc.clear();
    const int32_t* ptab = a.page_table + (size_t)r * a.maxp;
    const size_t head_bytes = (size_t)2 * 16 * HD;
    const uint8_t* base = a.c.codes + (size_t)kh * head_bytes;

    for (int ch = pg0; ch < pg1; ch += K8_IDS) {
        const int cnt = min(K8_IDS, pg1 - ch), steps = (cnt + 1) / 2;
        // lane i: page ch + i (-1: a hole, or past the split) and its scale bytes
        int id = lane < cnt ? ptab[ch + lane] : -1;
        if (id < 0 || id >= a.c.n_pages) id = -1;
        const uint32_t sc = id < 0 ? 0u : *reinterpret_cast<const uint16_t*>(a.c.scales + ((size_t)id * a.c.Hkv + kh) * 2);
        uint4 kb[2][H], vb[2][H];
        // K (side 0) or V of step s, into the operand registers; a hole reads page 0, unseen
        auto fetch = [&](int s, int side, uint4 (&x)[2][H]) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int pg = max(__builtin_amdgcn_readlane(id, 2 * s + e), 0);
                const uint8_t* p = base + (size_t)pg * a.c.Hkv * head_bytes + side * (16 * HD);
#pragma unroll
                for (int h = 0; h < H; ++h)
                    x[e][h] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_k8*>(p + h * 1024 + lane * 16)));
            }
        };
        if (wave < steps) {
            fetch(wave, 0, kb);
            fetch(wave, 1, vb);
        }
        for (int s = wave; s < steps; s += WAVES) {
            const bool more = s + WAVES < steps;
            float ksc[2], vsc[2];
            int mapped = 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t b = (uint32_t)__builtin_amdgcn_readlane((int)sc, 2 * s + e);
                ksc[e] = __uint_as_float((b & 0xffu) << 23);
                vsc[e] = __uint_as_float((b >> 8) << 23);
                mapped |= (__builtin_amdgcn_readlane(id, 2 * s + e) >= 0) << e;
            }
            const int j0 = 16 * (ch + 2 * s);
            const bool edge = mapped != 3 || j0 + 31 > row.p0 || j0 + 32 > row.len ||
                              (a.window && j0 <= k8_hidden(a.window, row.p0 + row.n - 1));
            float x[NT][8];
            k8_scores<HD, NT, CAP>(kb, ksc, qa, so, x);
            __builtin_amdgcn_sched_barrier(0);
            if (more) fetch(s + WAVES, 0, kb);  // its registers are free: in flight under the rest of the step
            __builtin_amdgcn_sched_barrier(0);
            if (edge) {
#pragma unroll
                for (int u = 0; u < NT; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        x[u][i] = k8_sees(row, a.window, j0, mapped, g, i, pc[u]) ? x[u][i] : -__builtin_inff();
            }
            bf16x8_k8 p[NT][2];
            k8_softmax<HD, NT, 2>(x, so.f, acc, p);
            if (edge) k8_mend_odd<HD, NT>(vb, vsc, acc, row, a.window, j0, mapped, g, pc);
            k8_pv<HD, NT, 2>(vb, vsc, p, acc);
            __builtin_amdgcn_sched_barrier(0);
            if (more) fetch(s + WAVES, 1, vb);
        }
    }

    // the waves' shares join in LDS
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const float ls = k8_col_sum(acc.l[u]);
        if (g == 0) {
            sh.m[wave][16 * u + c] = acc.m[u];
            sh.l[wave][16 * u + c] = ls;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
            *reinterpret_cast<f32x4_k8*>(&sh.o[wave][16 * u + c][16 * d + 4 * g]) = acc.o[u][d];
    }
    __syncthreads();
    const int live = row.n * a.G;
    for (int i = threadIdx.x; i < live * (HD / 4); i += 64 * WAVES) {
        const int rr = i / (HD / 4), d = i % (HD / 4) * 4;
        float M = sh.m[0][rr];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sh.m[w][rr]);
        float L = 0.0f;
        f32x4_k8 O = f32x4_k8{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(sh.m[w][rr] - M);
            L += f * sh.l[w][rr];
            O += f * *reinterpret_cast<const f32x4_k8*>(&sh.o[w][rr][d]);
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
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(NT == 2 || WAVES > 4 ? 2 : 3))) void attn_kv8_few_kernel(
    Kv8AttnArgs a, K8Few few) {
    __shared__ __attribute__((aligned(16))) K8FewShared<HD, NT, WAVES> sh;
    k8_few_block<HD, NT, WAVES, CAP, EVEN>(a, few, blockIdx.x, sh);
}

// One query row's splits joined in their order by a wave: outputs at po + s * so, reference and sum of split s in lane s's
// ml (act <= 64).
template <int HD>
__device__ __forceinline__ void k8_join(const float* po, size_t so, const float* pml, size_t sml, int act, uint16_t* out) {
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
    const float f = lane < act ? __builtin_amdgcn_exp2f(ml.x - M) : 0.0f;
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

// Joins the splits of rows of few query rows: a wave per query row of a (row, KV head); block: its index, of ROWB blocks a
// (row, KV head).
template <int HD, int NT, bool EVEN>
__device__ __forceinline__ void k8_few_join(const Kv8AttnArgs& a, const K8Few& few, int block, int rowb) {
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
    k8_join<HD>(a.part + first * HD, (size_t)(16 * NT) * HD, ml + 2 * first, 2 * 16 * NT, act, k8_out(a, row, kh, rr));
}
template <int HD, int NT, bool EVEN>
__global__ __launch_bounds__(K8_THREADS) void attn_kv8_join_kernel(Kv8AttnArgs a, K8Few few, int rowb) {
    k8_few_join<HD, NT, EVEN>(a, few, blockIdx.x, rowb);
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
constexpr int K8_STAGE = 4;       // pages a stage of the chunk kernel, one a wave to fetch
constexpr int K8_MIN_STAGES = 4;  // stages a split of a tile takes at least
constexpr int K8_CHUNK_TILES = 2; // tiles of 16 query rows a wave of a chunk's block holds
constexpr int K8_CHUNK_ROWS = K8_WAVES * 16 * K8_CHUNK_TILES;
// The pages that tile t's tokens see, the stages of four pages they make and the splits that share these.
struct K8Span {
    int pg0, pg1, stages, act;
};
template <int ROWS>
__device__ __forceinline__ K8Span k8_span(const Kv8AttnArgs& a, const K8Row& row, int t, int nsplit) {
    const int p0 = row.p0 + t * ROWS / a.G, p1 = row.p0 + (min((t + 1) * ROWS, row.n * a.G) - 1) / a.G;
    K8Span x;
    x.pg0 = a.window ? min(k8_hidden(a.window, p0) + 1, row.len) / 16 : 0;
    x.pg1 = max(0, min(p1 + 1, row.len) + 15) / 16;
    x.stages = max(0, (x.pg1 - x.pg0 + K8_STAGE - 1) / K8_STAGE);
    x.act = max(1, min(nsplit, x.stages / K8_MIN_STAGES));
    return x;
}

// Rows of more query rows: one block of 8 waves per (row, KV head, 64 NT query rows, split of the positions that these see),
// the tokens of a row's end first (they see the most).  Bound by the matrix cores (37 % busy) and the vector units (47 %),
// which hardly work at once: a product of 16x16x32 alone takes 20.6 cycles, with four vector instructions beside it most of
// their sum, from two waves as from one.  The waves form two groups of four; a wave holds NT
// tiles of query rows, the same in both groups, and each group takes half of the block's positions in stages of 4
// pages, which go through a double buffer of the group's in LDS as bf16 matrix operands: a wave fetches and
// converts one page, so that a code is converted once a group and an operand is one read for NT products.  The
// next stage is in flight in registers while one is used, and one barrier a stage parts them.  A wave alone
// on its SIMD leaves it idle for more than half of a stage (LDS reads, the chain from scores to probabilities): the
// two groups fill each other's gaps, and halve the time of the longest block.
constexpr int K8_GROUPS = 2;
constexpr int K8_CHUNK_THREADS = K8_GROUPS * K8_THREADS;
template <int HD>
struct K8ChunkShared {
    // operands of two stages, 16 bytes a lane: [stage][pair of pages][K: (page, h, half); V: output tile]
    uint32_t tile[K8_GROUPS][2][2][2][HD / 16][64][4];
    uint32_t odd_at[K8_GROUPS][2][K8_STAGE][64];  // codes of V that are not finite: bits 4 d .. of a lane: output tile d's four positions of a page
    int odd_any[K8_GROUPS][2][K8_STAGE];
};
template <int HD, int NT, bool CAP>
__device__ __forceinline__ void k8_chunk_block(const Kv8AttnArgs& a, int few, int tiles, int nsplit, float* part, int block,
                                               K8ChunkShared<HD>& sh) {
    constexpr int H = HD / 64, DT = HD / 16;
    constexpr int ROWS = K8_WAVES * 16 * NT;
    static_assert(NT * DT * 4 * K8_THREADS <= sizeof(sh.tile) / K8_GROUPS / 4, "a group's outputs fit its tiles");
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / K8_THREADS);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % K8_WAVES;
    const int kh = block % a.c.Hkv;
    uint32_t(*tile)[2][2][DT][64][4] = sh.tile[group];
    uint32_t(*odd_at)[K8_STAGE][64] = sh.odd_at[group];
    int(*odd_any)[K8_STAGE] = sh.odd_any[group];
    const int split = block / a.c.Hkv % nsplit, index = block / a.c.Hkv / nsplit;
    const K8Tile at = k8_tile<ROWS>(a, few, index);
    if (at.r < 0) return;
    const int r = __builtin_amdgcn_readfirstlane(at.r), t = __builtin_amdgcn_readfirstlane(at.t);
    const K8Row row = k8_row(a, r);
    const int live = row.n * a.G;
    if (t * ROWS >= live) return;
    K8Span span = k8_span<ROWS>(a, row, t, nsplit);
    if (split >= span.act) return;
    // the block's stages, and the group's of them; most: those of the group that has more
    const int b0 = span.stages * split / span.act, b1 = span.stages * (split + 1) / span.act, half = (b0 + b1 + 1) / 2;
    const int st0 = group ? half : b0, stages = (group ? b1 : half) - st0, most = half - b0;
    const int pg0 = span.pg0 + st0 * K8_STAGE, pg1 = min(span.pg1, pg0 + stages * K8_STAGE);
    // the positions of the wave's tokens
    const int rr0 = t * ROWS + wave * (16 * NT);
    const int wp0 = row.p0 + min(rr0, live - 1) / a.G, wp1 = row.p0 + (min(rr0 + 16 * NT, live) - 1) / a.G;

    uint4 qa[NT][2 * H];
    int pc[NT];
    k8_query<HD, NT>(a, row, kh, rr0, c, g, qa, pc);
    const K8Soft so = k8_soft(a);
    K8Acc<HD, NT> acc;
    acc.clear();
    uint32_t odd_out[NT];  // bit 4 d + i: output i of tile d saw a value of V that is not finite
#pragma unroll
    for (int u = 0; u < NT; ++u) odd_out[u] = 0;
    const int32_t* ptab = a.page_table + (size_t)r * a.maxp;
    const size_t head_bytes = (size_t)2 * 16 * HD;
    const uint8_t* base = a.c.codes + (size_t)kh * head_bytes;

    // lane i: page pg0 + 64 k + i of the table (-1: not one of the cache's, or past the group's), of the 64 that hold the
    // stage fetched last, and its scale bytes; and the next 64's
    auto page_id = [&](int i) {
        return i < pg1 ? *reinterpret_cast<const int32_t*>(reinterpret_cast<const char*>(ptab) + 4u * (uint32_t)i) : -1;
    };
    auto valid = [&](int v) { return v < 0 || v >= a.c.n_pages ? -1 : v; };
    auto scale_bytes = [&](int v) {
        return v < 0 ? 0u : (uint32_t) * reinterpret_cast<const uint16_t*>(a.c.scales + ((size_t)v * a.c.Hkv + kh) * 2);
    };
    int id = -1, idn = valid(page_id(pg0 + lane));
    uint32_t sc = 0, scn = scale_bytes(idn);
    // the wave's page of the next stage: K, V, their scales, and which of the stage's pages are mapped
    u32x4_k8 nx[2][H];
    float nsc[2];
    int map = 0;
    const size_t page_bytes = (size_t)a.c.Hkv * head_bytes;
    auto fetch = [&](int st, u32x4_k8 (&x)[2][H], float (&xs)[2], int& m, int& id, uint32_t& sc, int& idn, uint32_t& scn) {
        const int at = st * K8_STAGE % K8_IDS;
        if (at == 0) {
            id = idn;
            sc = scn;
            idn = page_id(pg0 + st * K8_STAGE + K8_IDS + lane);
        }
        if (at == K8_IDS / 2) {  // halfway: the next ids are there, their scales are requested
            idn = valid(idn);
            scn = scale_bytes(idn);
        }
        m = (int)(__ballot(id >= 0) >> at) & 15;
        const int mine = at + wave;
        const uint32_t b = (uint32_t)__builtin_amdgcn_readlane((int)sc, mine);
        xs[0] = __uint_as_float((b & 0xffu) << 23);
        xs[1] = __uint_as_float(b >> 8 << 23);
        const uint64_t p = k8_uniform(base + (size_t)max(__builtin_amdgcn_readlane(id, mine), 0) * page_bytes);
#pragma unroll
        for (int h = 0; h < 2 * H; ++h) x[h / H][h % H] = k8_load(p, h * 1024u + lane * 16u);
    };
    auto put = [&](int buf, const u32x4_k8 (&x)[2][H], const float (&xs)[2]) {
        const int pair = wave >> 1, e = wave & 1;
        const uint32_t add = k8_odd_add(xs[1]);
        uint32_t any = 0;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) any |= (x[1][h][q] & 0x7f7f7f7fu) + add;
        const bool some = __any((any & 0x80808080u) != 0);
        if (lane == 0) odd_any[buf][wave] = some;
        uint32_t at = 0;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
                const uint2 lo = k8_bf16x4(x[0][h][q], xs[0]), hi = k8_bf16x4(x[0][h][q + 1], xs[0]);
                *reinterpret_cast<u32x4_k8*>(tile[buf][pair][0][(e * H + h) * 2 + (q >> 1)][lane]) = u32x4_k8{lo.x, lo.y, hi.x, hi.y};
            }
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint2 w = k8_bf16x4(x[1][h][q], xs[1]);
                *reinterpret_cast<u32x2_k8*>(&tile[buf][pair][1][4 * h + q][lane][2 * e]) = u32x2_k8{w.x, w.y};
            }
        if (some) {  // codes that are not finite are noted, and their operands become 0
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t b = k8_odd_bytes(x[1][h][q], add) >> 7;  // bits 0, 8, 16, 24
                    at |= ((b | b >> 7 | b >> 14 | b >> 21) & 15u) << (4 * (4 * h + q));
                    uint32_t* w = &tile[buf][pair][1][4 * h + q][lane][2 * e];
                    w[0] &= ~((b & 1u) * 0xffffu | (b >> 8 & 1u) * 0xffff0000u);
                    w[1] &= ~((b >> 16 & 1u) * 0xffffu | (b >> 24) * 0xffff0000u);
                }
            odd_at[buf][wave][lane] = at;
        }
    };
    // The second group's waves go first where both could issue: the groups meet at every barrier, and would
    // else want the matrix cores and the vector units at the same times (a prompt of 4000 tokens, 40 heads over 8: 220 us, 209 so)
    if (group) __builtin_amdgcn_s_setprio(1);
    int now = 0;
    if (stages) {
        fetch(0, nx, nsc, map, id, sc, idn, scn);
        put(0, nx, nsc);
    }
    for (int st = 0; st < most; ++st) {
        const int buf = st & 1;
        now = map;
        __syncthreads();
        if (st < stages) {  // (else the last stage is the other group's alone)
        // K's operands of the first 32 positions; V's are requested before the softmax and K's of the second 32
        // before V's product, so that an operand is waited for only where its latency has passed under other work
        bf16x8_k8 kf[4 * H], vf[DT];
        auto read_k = [&](int hf, int e, bf16x8_k8 (&kf)[4 * H]) {
#pragma unroll
            for (int k = 2 * H * e; k < 2 * H * (e + 1); ++k) kf[k] = *reinterpret_cast<const bf16x8_k8*>(tile[buf][hf][0][k][lane]);
        };
        read_k(0, 0, kf);
        read_k(0, 1, kf);
        const int bad[2] = {odd_any[buf][0] | odd_any[buf][1], odd_any[buf][2] | odd_any[buf][3]};
        __builtin_amdgcn_sched_barrier(0);
        if (st + 1 < stages) fetch(st + 1, nx, nsc, map, id, sc, idn, scn);
#pragma unroll
        for (int hf = 0; hf < K8_STAGE / 2; ++hf) {
            const int j0 = 16 * (pg0 + st * K8_STAGE) + 32 * hf;
            // whether there is anything for this wave's tokens in these 32 positions
            const bool any = j0 <= wp1 && !(a.window && j0 + 31 <= k8_hidden(a.window, wp0));
            const int mapped = now >> (2 * hf) & 3;
            const bool edge = mapped != 3 || j0 + 31 > wp0 || j0 + 32 > row.len || (a.window && j0 <= k8_hidden(a.window, wp1));
            if (hf == 1) {
                read_k(1, 1, kf);
                __builtin_amdgcn_sched_barrier(0);
            }
            float x[NT][8];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                f32x4_k8 s[NT];
#pragma unroll
                for (int u = 0; u < NT; ++u) s[u] = f32x4_k8{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < 2 * H; ++k)
#pragma unroll
                    for (int u = 0; u < NT; ++u)
                        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[e * 2 * H + k], __builtin_bit_cast(bf16x8_k8, qa[u][k]), s[u], 0, 0, 0);
#pragma unroll
                for (int u = 0; u < NT; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[u][4 * e + i] = s[u][i];
            }
            if (CAP && any) k8_cap<NT>(x, so);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int d = 0; d < DT; ++d) vf[d] = *reinterpret_cast<const bf16x8_k8*>(tile[buf][hf][1][d][lane]);
            __builtin_amdgcn_sched_barrier(0);
            bf16x8_k8 p[NT][1];
            if (any) {
                if (edge) {
#pragma unroll
                    for (int u = 0; u < NT; ++u)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            x[u][i] = k8_sees(row, a.window, j0, mapped, g, i, pc[u]) ? x[u][i] : -__builtin_inff();
                }
                k8_softmax<HD, NT, 1>(x, so.f, acc, p);
            }
            if (any && bad[hf]) {
                // V's codes that are not finite went into the tile as 0: a product of the codes' and the columns' indicators finds the
                // outputs that see one, which become NaN at the end
                // (tile by tile of query rows, the codes' indicators made anew for each: 32 registers less)
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    uint32_t n[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        n[e] = odd_any[buf][2 * hf + e] ? odd_at[buf][2 * hf + e][lane] : 0u;
                        asm("" : "+v"(n[e]));
                    }
                    u32x4_k8 sw;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sw[i] = (k8_sees(row, a.window, j0, mapped, g, 2 * i, pc[u]) ? 0x3f80u : 0u) |
                                (k8_sees(row, a.window, j0, mapped, g, 2 * i + 1, pc[u]) ? 0x3f800000u : 0u);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        __builtin_amdgcn_sched_barrier(0);
                        u32x4_k8 f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t b = n[i >> 1] >> (4 * d + 2 * (i & 1));
                            f[i] = (b & 1u ? 0x3f80u : 0u) | (b & 2u ? 0x3f800000u : 0u);
                        }
                        f32x4_k8 hit = f32x4_k8{0.f, 0.f, 0.f, 0.f};
                        hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_k8, f), __builtin_bit_cast(bf16x8_k8, sw), hit, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t one = hit[i] > 0.0f ? 1u : 0u;
                            asm("" : "+v"(one));  // (shifted, not chosen from 32 constants that would take registers)
                            odd_out[u] |= one << (4 * d + i);
                        }
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (hf == 0) read_k(1, 0, kf);  // (the second page's when V's registers are free)
            __builtin_amdgcn_sched_barrier(0);
            if (!any) continue;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int u = 0; u < NT; ++u) acc.o[u][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[d], p[u][0], acc.o[u][d], 0, 0, 0);
        }
        if (st + 1 < stages) put(buf ^ 1, nx, nsc);
        }
    }
    // the second group's outputs join the first's, through its own tiles
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        acc.l[u] = k8_col_sum(acc.l[u]);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (odd_out[u] >> (4 * d + i) & 1u) acc.o[u][d][i] = __builtin_nanf("");
    }
    __syncthreads();
    f32x4_k8* other = reinterpret_cast<f32x4_k8*>(sh.tile[1]) + wave * (NT * DT * 64) + lane;
    float* other_ml = reinterpret_cast<float*>(sh.tile[0]) + wave * (2 * NT * 64) + lane;
    if (group) {
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            other_ml[2 * u * 64] = acc.m[u];
            other_ml[(2 * u + 1) * 64] = acc.l[u];
#pragma unroll
            for (int d = 0; d < DT; ++d) other[(u * DT + d) * 64] = acc.o[u][d];
        }
    }
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const float m1 = other_ml[2 * u * 64], M = fmaxf(acc.m[u], m1);
        const float f0 = __builtin_amdgcn_exp2f(acc.m[u] - M), f1 = __builtin_amdgcn_exp2f(m1 - M);
        acc.m[u] = M;
        acc.l[u] = acc.l[u] * f0 + other_ml[(2 * u + 1) * 64] * f1;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc.o[u][d] = acc.o[u][d] * f0 + other[(u * DT + d) * 64] * f1;
        const float L = acc.l[u];
        const float inv = L == 0.0f ? 0.0f : ieee_div(1.0f, L);
        const int rr = rr0 + 16 * u + c;
        if (rr >= live) continue;
        if (span.act > 1) {
            const size_t pr = ((size_t)(index * a.c.Hkv + kh) * nsplit + split) * ROWS + wave * (16 * NT) + 16 * u + c;
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4_k8*>(part + pr * HD + 16 * d + 4 * g) = acc.o[u][d];
            if (g == 0) {
                float* ml = part + (size_t)tiles * a.c.Hkv * nsplit * ROWS * HD + 2 * pr;
                ml[0] = acc.m[u];
                ml[1] = L;
            }
            continue;
        }
        uint16_t* out = k8_out(a, row, kh, rr) + 4 * g;
#pragma unroll
        for (int d = 0; d < DT; ++d)
            *reinterpret_cast<uint2*>(out + 16 * d) =
                make_uint2(k8_pack(acc.o[u][d][0] * inv, acc.o[u][d][1] * inv), k8_pack(acc.o[u][d][2] * inv, acc.o[u][d][3] * inv));
    }
}

// A call with longer rows: their blocks, then those of its rows of few query rows, in one launch.
template <int HD, bool CAP>
__global__ __launch_bounds__(K8_CHUNK_THREADS) __attribute__((amdgpu_waves_per_eu(2))) void attn_kv8_mixed_kernel(
    Kv8AttnArgs a, K8Few few, int tiles, int csplit, float* cpart) {
    union Shared {
        K8ChunkShared<HD> chunk;
        K8FewShared<HD, 1, K8_GROUPS * K8_WAVES> few;
    };
    __shared__ __attribute__((aligned(16))) Shared sh;
    const int chunks = tiles * a.c.Hkv * csplit;
    if ((int)blockIdx.x < chunks)
        k8_chunk_block<HD, K8_CHUNK_TILES, CAP>(a, 16, tiles, csplit, cpart, blockIdx.x, sh.chunk);
    else
        k8_few_block<HD, 1, K8_GROUPS * K8_WAVES, CAP, false>(a, few, blockIdx.x - chunks, sh.few);
}

// Joins the splits of attn_kv8_mixed_kernel: blocks of its longer rows' tiles (csplit > 1), a wave per query row, then of the
// others.
template <int HD>
__global__ __launch_bounds__(K8_THREADS) void attn_kv8_mixed_join_kernel(Kv8AttnArgs a, K8Few few, int rowb, int tiles, int csplit,
                                                                        const float* cpart) {
    constexpr int ROWS = K8_CHUNK_ROWS, RB = ROWS / K8_WAVES;
    const int chunks = csplit > 1 ? tiles * a.c.Hkv * RB : 0;
    if ((int)blockIdx.x >= chunks) {
        k8_few_join<HD, 1, false>(a, few, blockIdx.x - chunks, rowb);
        return;
    }
    const int at = blockIdx.x / RB, kh = at % a.c.Hkv;
    const K8Tile tile = k8_tile<ROWS>(a, 16, at / a.c.Hkv);
    if (tile.r < 0) return;
    const K8Row row = k8_row(a, tile.r);
    const int i = blockIdx.x % RB * K8_WAVES + (threadIdx.x >> 6), rr = tile.t * ROWS + i;
    if (rr >= row.n * a.G) return;
    const int act = k8_span<ROWS>(a, row, tile.t, csplit).act;
    if (act == 1) return;
    const size_t first = (size_t)at * csplit * ROWS + i;
    const float* ml = cpart + (size_t)tiles * a.c.Hkv * csplit * ROWS * HD;
    k8_join<HD>(cpart + first * HD, (size_t)ROWS * HD, ml + 2 * first, 2 * ROWS, act, k8_out(a, row, kh, rr));
}

// The launch.  Measured on graphs of calls, 32 query heads over 8 KV heads of 128 where nothing else is said, us.
// Calls of rows of few query rows:
//   - rows are split until two blocks a CU are there (one: 23 rows of four tokens, 28 heads over 4, 27.9 -> 34.8; three: 64
//     rows of 512..768, 512 blocks without a split, 18.9 -> 24.1, as the join is a launch of its own; four: 23 rows
//     of four tokens 34.3, 40 rows of three 44.9 -> 40.7);
//   - a split takes at most 128 pages (64: 32 rows of 4096..16384 122 -> 125, 128 ragged rows 60.4 -> 59.2;
//     256: 122 -> 134);
//   - where the blocks of unsplit rows fit the device at once and a row has few pages, one block of 8
//     waves takes a row whole: one row of 512 7.1 -> 6.3, 32 rows of 512 12.1 -> 9.8; at 64 pages one row
//     7.9 -> 9.7, but 32 rows 17.0 -> 14.7, so up to 32 pages, or 64 where the blocks are half of the CUs.
//   - the host knows only the longest row; where a split takes 64 pages or more and a wave's lanes hold the rows (2 to 64), the
//     blocks find from all lengths how few pages fill the same number of blocks (16 rows of 16..16000, 28 heads
//     over 4: 37.1 -> 34.5, 40 of 16..7000 62.4 -> 57.6, 8 of four tokens behind 500..16000 37.6 -> 35.7; it takes a microsecond, so
//     with small splits it loses: 8 rows of 1000 10.1 -> 11.6).
// Calls with longer rows:
//   - a row of few query rows is split at 256 pages, beside the chunks' blocks, which take as long (64: 8 rows of
//     16000 beside a chunk of 512 57.8 -> 63.5, 30 of 4000 55.4 -> 63.2; no split: 103, 55.2), at 128 where
//     these rows' blocks are an eighth of the CUs (a row of 16000 beside two chunks of 64 tokens 35.7 -> 26.2);
//   - a tile of a chunk is split over its positions until there is a block a CU (two: one chunk of 64 behind 16000
//     tokens 45.9 -> 55.1, one of 512 behind 512 27.0 -> 45.1, no call faster: a CU holds one block, and the splits'
//     outputs are written and read), down to 4 stages a split (2: no difference; 8: 4 chunks of 2048 579 -> 600).
struct K8Plan {
    int nt, waves;              // rows of few query rows: tiles and waves of a block
    K8Few few;                  // and how they are split
    int64_t few_blocks;
    int64_t tiles;              // of 128 query rows, of the longer rows: at most (a row's last may be partly empty); 0: none
    int csplit;                 // splits of such a tile
};
constexpr int K8_MAX_PAGES = 128;
constexpr int K8_MAX_SPLITS = 64;
constexpr int K8_BLOCKS_PER_CU = 2;
constexpr int K8_WHOLE_PAGES = 32;
constexpr int K8_EVEN_PAGES = 64;
constexpr int K8_MIXED_PAGES = 256;
constexpr int K8_CHUNK_BLOCKS_PER_CU = 1;
// pages that a group of `tokens` neighbouring tokens of a row sees at most, by the host's bounds
static int64_t k8_pages(const Kv8AttnArgs& a, int64_t tokens) {
    int64_t len = a.max_len;
    if (a.window) len = std::min<int64_t>(len, (int64_t)a.window + tokens + 15);
    return std::max<int64_t>(1, (len + 15) / 16);
}
static K8Plan k8_plan(const Kv8AttnArgs& a) {
    K8Plan p;
    const int64_t rows = (int64_t)a.max_new * a.G;
    p.tiles = rows <= 32 ? 0 : (int64_t)a.T * a.G / K8_CHUNK_ROWS + std::min(a.B, a.T);
    p.nt = rows <= 16 || p.tiles ? 1 : 2;
    const int64_t pages = k8_pages(a, std::min(a.max_new, 16 * p.nt / a.G));
    const int64_t blocks = (int64_t)a.B * a.c.Hkv;
    const int64_t want = std::max<int64_t>(1, (K8_BLOCKS_PER_CU * a.n_cu + blocks / 2) / blocks);
    int64_t sp = std::min<int64_t>(K8_MAX_PAGES, std::max<int64_t>(K8_MIN_PAGES, (pages + want - 1) / want));
    if (p.tiles) sp = std::min<int64_t>(8 * blocks <= a.n_cu ? K8_MIXED_PAGES / 2 : K8_MIXED_PAGES, pages);
    sp = std::max(sp, (pages + K8_MAX_SPLITS - 1) / K8_MAX_SPLITS);
    p.waves = K8_WAVES;
    if (p.nt == 1 && blocks <= a.n_cu && pages <= (2 * blocks >= a.n_cu ? 2 : 1) * K8_WHOLE_PAGES) {
        p.waves = 2 * K8_WAVES;
        sp = pages;
    }
    const int nsplit = (int)((pages + sp - 1) / sp);
    const int units = K8_BLOCKS_PER_CU * a.n_cu / a.c.Hkv;
    p.few = K8Few{(int)sp, nsplit, nsplit, 0};
    p.few_blocks = blocks * nsplit;
    if (!p.tiles && nsplit > 1 && sp >= K8_EVEN_PAGES && a.B > 1 && a.B <= 64 && a.B < units && (int64_t)a.B * a.maxp <= 1 << 30) {
        p.few.most = std::min(2 * nsplit, K8_MAX_SPLITS);
        p.few.units = units;
        p.few_blocks = std::max<int64_t>(p.few_blocks, (int64_t)units * a.c.Hkv);
    }
    p.csplit = 1;
    if (p.tiles) {
        const int64_t stages = (k8_pages(a, std::min(a.max_new, K8_CHUNK_ROWS / a.G + 1)) + K8_STAGE - 1) / K8_STAGE;
        const int64_t most = std::min<int64_t>(K8_MAX_SPLITS, std::max<int64_t>(1, stages / K8_MIN_STAGES));
        p.csplit = (int)std::min<int64_t>(most, std::max<int64_t>(1, K8_CHUNK_BLOCKS_PER_CU * a.n_cu / (p.tiles * a.c.Hkv)));
    }
    return p;
}

static size_t k8_few_floats(const Kv8AttnArgs& a, const K8Plan& p) {
    return p.few.nsplit == 1 ? 0 : (size_t)a.B * a.c.Hkv * p.few.most * (16 * p.nt) * (a.c.hd + 2);
}
size_t kv8_attention_ws_bytes(const Kv8AttnArgs& a) {
    const K8Plan p = k8_plan(a);
    const size_t chunk = p.csplit == 1 ? 0 : (size_t)p.tiles * a.c.Hkv * p.csplit * K8_CHUNK_ROWS * (a.c.hd + 2);
    return (k8_few_floats(a, p) + chunk) * sizeof(float);
}

template <int HD, int NT, int WAVES, bool EVEN>
static void k8_launch_few(const Kv8AttnArgs& a, const K8Plan& p, int rowb, int64_t joins, hipStream_t s) {
    auto f = a.cap > 0.0f ? attn_kv8_few_kernel<HD, NT, WAVES, true, EVEN> : attn_kv8_few_kernel<HD, NT, WAVES, false, EVEN>;
    hipLaunchKernelGGL(f, dim3((unsigned)p.few_blocks), dim3(64 * WAVES), 0, s, a, p.few);
    if (joins)
        hipLaunchKernelGGL((attn_kv8_join_kernel<HD, NT, EVEN>), dim3((unsigned)joins), dim3(K8_THREADS), 0, s, a, p.few, rowb);
}
template <int HD>
static void k8_launch(const Kv8AttnArgs& a, const K8Plan& p, hipStream_t s) {
    const int rowb = (int)(std::min<int64_t>((int64_t)a.max_new * a.G, 16 * p.nt) + K8_WAVES - 1) / K8_WAVES;
    const int64_t few_joins = p.few.nsplit > 1 ? (int64_t)a.B * a.c.Hkv * rowb : 0;
    if (p.tiles == 0) {
        auto f = p.nt == 2 ? (p.few.units ? k8_launch_few<HD, 2, K8_WAVES, true> : k8_launch_few<HD, 2, K8_WAVES, false>)
                 : p.waves == K8_WAVES ? (p.few.units ? k8_launch_few<HD, 1, K8_WAVES, true> : k8_launch_few<HD, 1, K8_WAVES, false>)
                                       : k8_launch_few<HD, 1, 2 * K8_WAVES, false>;
        f(a, p, rowb, few_joins, s);
        return;
    }
    float* cpart = a.part + k8_few_floats(a, p);
    const dim3 grid((unsigned)(p.tiles * a.c.Hkv * p.csplit + p.few_blocks));
    auto f = a.cap > 0.0f ? attn_kv8_mixed_kernel<HD, true> : attn_kv8_mixed_kernel<HD, false>;
    hipLaunchKernelGGL(f, grid, dim3(K8_CHUNK_THREADS), 0, s, a, p.few, (int)p.tiles, p.csplit, cpart);
    const int64_t joins = few_joins + (p.csplit > 1 ? p.tiles * a.c.Hkv * (K8_CHUNK_ROWS / K8_WAVES) : 0);
    if (joins)
        hipLaunchKernelGGL(attn_kv8_mixed_join_kernel<HD>, dim3((unsigned)joins), dim3(K8_THREADS), 0, s, a, p.few, rowb,
                           (int)p.tiles, p.csplit, cpart);
}

bool kv8_attention_fits(const Kv8AttnArgs& a) {
    const K8Plan p = k8_plan(a);
    constexpr int64_t most = 1 << 22;  // blocks of a launch
    return (int64_t)a.T * a.G <= (1 << 29) && p.tiles * a.c.Hkv * p.csplit + p.few_blocks <= most &&
           (int64_t)a.B * a.c.Hkv * 8 + p.tiles * a.c.Hkv * (p.csplit > 1 ? K8_CHUNK_ROWS / K8_WAVES : 0) <= 2 * most;
}

hipError_t launch_kv8_attention(const Kv8AttnArgs& a, hipStream_t s) {
    const K8Plan p = k8_plan(a);
    if (a.c.hd == 128)
        k8_launch<128>(a, p, s);
    else
        k8_launch<64>(a, p, s);
    return hipGetLastError();
}

}  // namespace mg
