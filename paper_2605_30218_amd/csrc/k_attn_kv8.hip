// k_attn_kv8.hip -- attention of a batch's new tokens over the 8-bit paged K/V cache.
//
// One wave per (token, query head): a pass over the positions that the token sees with the running
// maximum, sum and output of the softmax, a lane holding hd / 64 features.
#include <algorithm>

#include "mg_device.h"
#include "mg_kernels.h"

namespace mg {

typedef __bf16 bf16x2_k8 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_k8 __attribute__((ext_vector_type(8)));
typedef float f32x4_k8 __attribute__((ext_vector_type(4)));

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
// high bit of every byte that is a NaN code
__device__ __forceinline__ uint32_t k8_nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

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
// <= p0 + i and, with a window, > p0 + i - window.
struct K8Row {
    int t0, n;      // its tokens of q
    int len, p0;    // positions in reach of the page table; position of its first token
    int pga, pgb;   // pages that any of its tokens sees: [pga, pgb)
};
__device__ __forceinline__ K8Row k8_row(const Kv8AttnArgs& a, int r) {
    K8Row x;
    x.t0 = a.cu_new ? min(max(a.cu_new[r], 0), a.T) : r;
    x.n = (a.cu_new ? min(a.cu_new[r + 1], a.T) : r + 1) - x.t0;
    const int len = a.lens[r];
    x.len = min(max(len, 0), 16 * a.maxp);
    x.p0 = len - x.n;
    x.pga = a.window ? max(0, min(x.p0 - a.window + 1, x.len)) / 16 : 0;
    x.pgb = (x.len + 15) / 16;
    return x;
}
// splits of npg pages among at most nsplit blocks of about sp pages (an even number each)
__device__ __forceinline__ int k8_active(int npg, int sp, int nsplit) {
    return min(nsplit, max(1, (npg + sp - 1) / sp));
}

// Rows of few query rows (tokens times query heads of a KV head <= 16 NT): one block of 4 waves per
// (row, KV head, split of the row's pages).
// A wave takes every 4th step of two pages and keeps the running maximum, sum and output of its share:
//   S^T[pos][c] = K[pos][:] . Q[c][:]      K the A operand, straight from the page: the cache stores a
//       head's page in the order in which a wave's 16-byte loads give the operand registers;
//   O^T[d][c] += V^T[d][pos] P^T[pos][c]   V the A operand, likewise; the scores' registers, positions
//       4 g .. 4 g + 3 of both pages in lane group g, are the B operand as they are.
// Column c of every product is one query row, in lanes c, c + 16, c + 32, c + 48, so its maximum is two
// exchanges and its rescaling a lane's own.  Codes become bf16 with their page's scale in one
// instruction a pair, exactly.  A probability is the sum of two bf16 terms (16 bits, 2^-16 of itself off),
// one product each: the matrix cores have the time, the K/V stream is what bounds the kernel.
template <int HD, int NT, bool CAP>
__global__ __launch_bounds__(K8_THREADS) __attribute__((amdgpu_waves_per_eu(NT == 1 ? 3 : 2))) void attn_kv8_few_kernel(Kv8AttnArgs a, int sp, int nsplit) {
    constexpr int H = HD / 64;        // 1 KiB runs of a page of K or V
    constexpr int DT = HD / 16;       // output tiles
    constexpr int OS = HD + 4;        // padded row of O in LDS
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kh = blockIdx.x % a.c.Hkv;
    const int r = blockIdx.x / a.c.Hkv % a.B, split = blockIdx.x / a.c.Hkv / a.B;
    const K8Row row = k8_row(a, r);
    if (row.n <= 0 || row.n * a.G > 16 * NT) return;
    const int npg = max(row.pgb - row.pga, 0);
    const int act = k8_active(npg, sp, nsplit);
    if (split >= act) return;
    const int per = ((npg + act - 1) / act + 1) & ~1;
    const int pg0 = row.pga + split * per, pg1 = split == act - 1 ? row.pgb : min(row.pgb, pg0 + per);

    __shared__ __attribute__((aligned(16))) float wo[K8_WAVES][16 * NT][OS];
    __shared__ float wm[K8_WAVES][16 * NT], wl[K8_WAVES][16 * NT];

    // query rows: tile u's column c is row 16 u + c = token * G + head of the KV head's group
    uint4 qa[NT][2 * H];
    int pc[NT];  // position of the column's token
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const int rr = 16 * u + c, tok = rr / a.G;
        const bool live = rr < row.n * a.G;
        const uint16_t* qp = a.q + (int64_t)(row.t0 + (live ? tok : 0)) * a.q_stride + (size_t)(kh * a.G + (live ? rr % a.G : 0)) * HD;
        pc[u] = row.p0 + (live ? tok : 0);
#pragma unroll
        for (int h = 0; h < H; ++h) {
            // operand slot (g, st) holds features 64 h + 16 g + 8 st ..
            qa[u][2 * h] = *reinterpret_cast<const uint4*>(qp + 64 * h + 16 * g);
            qa[u][2 * h + 1] = *reinterpret_cast<const uint4*>(qp + 64 * h + 16 * g + 8);
        }
    }
    const float sl2 = a.scale * 1.4426950408889634f;
    float m[NT], l[NT];
    f32x4_k8 o[NT][DT];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        m[u] = -__builtin_inff();
        l[u] = 0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[u][d] = f32x4_k8{0.f, 0.f, 0.f, 0.f};
    }
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
        // K (side 0) or V of step s, into the operand registers
        auto fetch = [&](int s, int side, uint4 (&x)[2][H]) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int pg = max(__builtin_amdgcn_readlane(id, 2 * s + e), 0);
                const uint8_t* p = base + (size_t)pg * a.c.Hkv * head_bytes + side * (16 * HD);
#pragma unroll
                for (int h = 0; h < H; ++h) x[e][h] = *reinterpret_cast<const uint4*>(p + h * 1024 + lane * 16);
            }
        };
        if (wave < steps) {
            fetch(wave, 0, kb);
            fetch(wave, 1, vb);
        }
        for (int s = wave; s < steps; s += K8_WAVES) {
            const bool more = s + K8_WAVES < steps;
            float ksc[2], vsc[2];
            bool hole = false;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t b = (uint32_t)__builtin_amdgcn_readlane((int)sc, 2 * s + e);
                ksc[e] = __uint_as_float((b & 0xffu) << 23);
                vsc[e] = __uint_as_float((b >> 8) << 23);
                hole |= __builtin_amdgcn_readlane(id, 2 * s + e) < 0;
            }
            const int j0 = 16 * (ch + 2 * s);
            const bool edge = hole || j0 + 31 > row.p0 || j0 + 32 > row.len ||
                              (a.window && j0 <= row.p0 + row.n - 1 - a.window);
            // scores, in log2 units: positions j0 + 16 e + 4 g + i of column c
            float x[NT][8];
            uint32_t see[NT];
#pragma unroll
            for (int u = 0; u < NT; ++u) see[u] = 0xffu;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                f32x4_k8 acc[NT];
#pragma unroll
                for (int u = 0; u < NT; ++u) acc[u] = f32x4_k8{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < H; ++h)
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
                    for (int i = 0; i < 4; ++i) {
                        if (CAP) {
                            // tanh(z) = 1 - 2 / (1 + e^2z)
                            const float z = acc[u][i] * a.scale * a.inv_cap;
                            const float t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * 2.8853900817779268f));
                            x[u][4 * e + i] = t * (a.cap * 1.4426950408889634f);
                        } else {
                            x[u][4 * e + i] = acc[u][i] * sl2;
                        }
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) fetch(s + K8_WAVES, 0, kb);  // its registers are free: in flight under the rest of the step
            __builtin_amdgcn_sched_barrier(0);
            if (edge) {
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    see[u] = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int j = j0 + 16 * (i >> 2) + 4 * g + (i & 3);
                        const bool mapped = __builtin_amdgcn_readlane(id, 2 * s + (i >> 2)) >= 0;
                        const bool v = mapped && j <= pc[u] && j < row.len && (!a.window || j > pc[u] - a.window);
                        x[u][i] = v ? x[u][i] : -__builtin_inff();
                        see[u] |= (uint32_t)v << i;
                    }
                }
            }
            bf16x8_k8 ph[NT], pl[NT];
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                float mx = fmaxf(fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3])),
                                 fmaxf(fmaxf(x[u][4], x[u][5]), fmaxf(x[u][6], x[u][7])));
                const float mn = fmaxf(m[u], k8_col_max(mx));
                const float ms = mn == -__builtin_inff() ? 0.0f : mn;
                const float al = __builtin_amdgcn_exp2f(m[u] - ms);
                m[u] = mn;
                float sum = 0.0f, lo[8];
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[u][i] = __builtin_amdgcn_exp2f(x[u][i] - ms);
                    sum += x[u][i];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = k8_pack(x[u][2 * i], x[u][2 * i + 1]);
                    lo[2 * i] = x[u][2 * i] - bf_lo(w[i]);
                    lo[2 * i + 1] = x[u][2 * i + 1] - bf_hi(w[i]);
                }
                l[u] = l[u] * al + sum;
                ph[u] = __builtin_bit_cast(bf16x8_k8, make_uint4(w[0], w[1], w[2], w[3]));
                pl[u] = __builtin_bit_cast(bf16x8_k8, make_uint4(k8_pack(lo[0], lo[1]), k8_pack(lo[2], lo[3]),
                                                                 k8_pack(lo[4], lo[5]), k8_pack(lo[6], lo[7])));
                if (__any(al != 1.0f)) {
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[u][d] *= al;
                }
            }
            // a NaN code of V under a probability of zero: in a step whose columns do not all see all
            // positions it must reach the columns that see it, and no other
            if (edge) {
                uint32_t any = 0;
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int h = 0; h < H; ++h)
                        any |= k8_nan_bytes(vb[e][h].x) | k8_nan_bytes(vb[e][h].y) | k8_nan_bytes(vb[e][h].z) | k8_nan_bytes(vb[e][h].w);
                if (__any(any != 0)) {
#pragma unroll
                    for (int h = 0; h < H; ++h)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint32_t* w[2] = {reinterpret_cast<uint32_t*>(&vb[0][h]) + q, reinterpret_cast<uint32_t*>(&vb[1][h]) + q};
                            uint32_t f[4];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const uint32_t nb = k8_nan_bytes(*w[e]);
                                *w[e] &= ~((nb >> 7) * 0xffu);
                                f[2 * e] = ((nb >> 7) & 1u) * 0x3f80u | ((nb >> 15) & 1u) * 0x3f800000u;
                                f[2 * e + 1] = ((nb >> 23) & 1u) * 0x3f80u | (nb >> 31) * 0x3f800000u;
                            }
                            const bf16x8_k8 F = __builtin_bit_cast(bf16x8_k8, make_uint4(f[0], f[1], f[2], f[3]));
#pragma unroll
                            for (int u = 0; u < NT; ++u) {
                                uint32_t sw[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    sw[i] = ((see[u] >> (2 * i)) & 1u) * 0x3f80u | ((see[u] >> (2 * i + 1)) & 1u) * 0x3f800000u;
                                f32x4_k8 hit = f32x4_k8{0.f, 0.f, 0.f, 0.f};
                                hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(F, __builtin_bit_cast(bf16x8_k8, make_uint4(sw[0], sw[1], sw[2], sw[3])), hit, 0, 0, 0);
#pragma unroll
                                for (int i = 0; i < 4; ++i) o[u][4 * h + q][i] = hit[i] > 0.0f ? __builtin_nanf("") : o[u][4 * h + q][i];
                            }
                        }
                }
            }
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t w0 = q == 0 ? vb[0][h].x : q == 1 ? vb[0][h].y : q == 2 ? vb[0][h].z : vb[0][h].w;
                    const uint32_t w1 = q == 0 ? vb[1][h].x : q == 1 ? vb[1][h].y : q == 2 ? vb[1][h].z : vb[1][h].w;
                    const uint2 lo = k8_bf16x4(w0, vsc[0]), hi = k8_bf16x4(w1, vsc[1]);
                    const bf16x8_k8 A = __builtin_bit_cast(bf16x8_k8, make_uint4(lo.x, lo.y, hi.x, hi.y));
#pragma unroll
                    for (int u = 0; u < NT; ++u) {
                        o[u][4 * h + q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, ph[u], o[u][4 * h + q], 0, 0, 0);
                        o[u][4 * h + q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, pl[u], o[u][4 * h + q], 0, 0, 0);
                    }
                }
            __builtin_amdgcn_sched_barrier(0);
            if (more) fetch(s + K8_WAVES, 1, vb);
        }
    }

    // the waves' shares join in LDS
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const float ls = k8_col_sum(l[u]);
        if (g == 0) {
            wm[wave][16 * u + c] = m[u];
            wl[wave][16 * u + c] = ls;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
            *reinterpret_cast<f32x4_k8*>(&wo[wave][16 * u + c][16 * d + 4 * g]) = o[u][d];
    }
    __syncthreads();
    const int live = row.n * a.G;
    for (int i = threadIdx.x; i < live * (HD / 4); i += K8_THREADS) {
        const int rr = i / (HD / 4), d = i % (HD / 4) * 4;
        float M = wm[0][rr];
#pragma unroll
        for (int w = 1; w < K8_WAVES; ++w) M = fmaxf(M, wm[w][rr]);
        const float Ms = M == -__builtin_inff() ? 0.0f : M;
        float L = 0.0f;
        f32x4_k8 O = f32x4_k8{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < K8_WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(wm[w][rr] - Ms);
            L += f * wl[w][rr];
            O += f * *reinterpret_cast<const f32x4_k8*>(&wo[w][rr][d]);
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

// Joins the splits of attn_kv8_few_kernel in their order: one block per (row, KV head), a wave a query row.
template <int HD, int NT>
__global__ __launch_bounds__(K8_THREADS) void attn_kv8_join_kernel(Kv8AttnArgs a, int sp, int nsplit) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int kh = blockIdx.x % a.c.Hkv, r = blockIdx.x / a.c.Hkv;
    const K8Row row = k8_row(a, r);
    const int live = row.n * a.G;
    if (row.n <= 0 || live > 16 * NT) return;
    const int act = k8_active(max(row.pgb - row.pga, 0), sp, nsplit);
    if (act == 1) return;
    const size_t first = ((size_t)r * a.c.Hkv + kh) * nsplit;
    const float* mls = a.part + (size_t)a.B * a.c.Hkv * nsplit * (16 * NT) * HD;
    for (int rr = wave; rr < live; rr += K8_WAVES) {
        // nsplit <= 64: lane s has split s
        const size_t at = (first + min(lane, act - 1)) * (16 * NT) + rr;
        const float2 ml = *reinterpret_cast<const float2*>(mls + 2 * at);
        const float ms = lane < act ? ml.x : -__builtin_inff();
        const float M = wave_max(ms);
        const float f = lane < act ? __builtin_amdgcn_exp2f(ms - (M == -__builtin_inff() ? 0.0f : M)) : 0.0f;
        const float L = wave_sum_fast(lane < act ? f * ml.y : 0.0f);
        const float inv = L == 0.0f ? 0.0f : ieee_div(1.0f, L);
        constexpr int PL = HD / 64;
        float O[PL];
#pragma unroll
        for (int e = 0; e < PL; ++e) O[e] = 0.0f;
        const float* po = a.part + (first * (16 * NT) + rr) * HD + PL * lane;
#pragma unroll 4
        for (int s = 0; s < act; ++s) {
            const float w = __shfl(f, s, 64);
#pragma unroll
            for (int e = 0; e < PL; ++e) O[e] += w * po[(size_t)s * (16 * NT) * HD + e];
        }
        uint16_t* out = a.out + (int64_t)(row.t0 + rr / a.G) * a.out_stride + (size_t)(kh * a.G + rr % a.G) * HD + PL * lane;
#pragma unroll
        for (int e = 0; e < PL; ++e) out[e] = (uint16_t)f2bf(O[e] * inv);
    }
}

// The launch of rows of few query rows: tiles a block holds, pages a split, splits of a row.
struct K8Plan {
    int nt, sp, nsplit;
};
constexpr int K8_MIN_PAGES = 8;    // pages a split takes at least: a step of every wave
constexpr int K8_MAX_PAGES = 64;
constexpr int K8_MAX_SPLITS = 64;
constexpr int K8_BLOCKS_PER_CU = 3;
static K8Plan k8_plan(const Kv8AttnArgs& a) {
    K8Plan p;
    p.nt = a.max_new * a.G <= 16 ? 1 : 2;
    int64_t len = a.max_len;
    if (a.window) len = std::min<int64_t>(len, (int64_t)a.window + a.max_new + 15);
    const int64_t pages = std::max<int64_t>(1, (len + 15) / 16);
    const int64_t blocks = (int64_t)a.B * a.c.Hkv;
    const int64_t want = std::max<int64_t>(1, (K8_BLOCKS_PER_CU * a.n_cu + blocks - 1) / blocks);
    int64_t sp = std::min<int64_t>(K8_MAX_PAGES, std::max<int64_t>(K8_MIN_PAGES, (pages + want - 1) / want));
    sp = std::max(sp, (pages + K8_MAX_SPLITS - 1) / K8_MAX_SPLITS);
    p.sp = (int)sp;
    p.nsplit = (int)((pages + sp - 1) / sp);
    return p;
}

size_t kv8_attention_ws_bytes(const Kv8AttnArgs& a) {
    const K8Plan p = k8_plan(a);
    return p.nsplit == 1 ? 0 : (size_t)a.B * a.c.Hkv * p.nsplit * (16 * p.nt) * (a.c.hd + 2) * sizeof(float);
}

template <int HD, int NT>
static hipError_t k8_few(const Kv8AttnArgs& a, const K8Plan& p, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)a.B * a.c.Hkv * p.nsplit));
    if (a.cap > 0.0f)
        hipLaunchKernelGGL((attn_kv8_few_kernel<HD, NT, true>), grid, dim3(K8_THREADS), 0, s, a, p.sp, p.nsplit);
    else
        hipLaunchKernelGGL((attn_kv8_few_kernel<HD, NT, false>), grid, dim3(K8_THREADS), 0, s, a, p.sp, p.nsplit);
    if (p.nsplit > 1)
        hipLaunchKernelGGL((attn_kv8_join_kernel<HD, NT>), dim3(a.B * a.c.Hkv), dim3(K8_THREADS), 0, s, a, p.sp, p.nsplit);
    return hipGetLastError();
}

__global__ __launch_bounds__(256) void attn_kv8_kernel(Kv8AttnArgs a, int few) {
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = (int)(w / a.Hq), head = (int)(w % a.Hq), kh = head / a.G, hd = a.c.hd;
    if (t >= a.T) return;
    int r = t, t0 = t, n = 1;
    if (a.cu_new) {
        int lo = 0, hi = a.B;  // the last row that begins at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.cu_new[mid] <= t) lo = mid; else hi = mid;
        }
        r = lo;
        t0 = a.cu_new[r];
        n = a.cu_new[r + 1] - t0;
        if (t < t0 || t >= t0 + n) return;
    }
    if (n * a.G <= few) return;
    const int len = min(a.lens[r], 16 * a.maxp), p = a.lens[r] - n + (t - t0);
    const int j1 = min(p + 1, len), j0 = a.window ? max(0, p - a.window + 1) : 0;
    const int per = hd / 64;
    const uint16_t* q = a.q + t * a.q_stride + head * hd;
    float qv[2], o[2] = {0.f, 0.f}, m = -__builtin_inff(), l = 0.f;
    for (int e = 0; e < per; ++e) qv[e] = bf2f(q[64 * e + lane]) * a.scale;
    for (int j = j0; j < j1; ++j) {
        const int pg = a.page_table[(size_t)r * a.maxp + j / 16];
        if (pg < 0 || pg >= a.c.n_pages) continue;
        const size_t ph = ((size_t)pg * a.c.Hkv + kh) * 2;
        const uint8_t* kp = a.c.codes + ph * (size_t)(16 * hd);
        const uint8_t* vp = kp + 16 * hd;
        const float ksc = __uint_as_float((uint32_t)a.c.scales[ph] << 23);
        const float vsc = __uint_as_float((uint32_t)a.c.scales[ph + 1] << 23);
        const int i = j % 16;
        float s = 0.f, v[2];
        for (int e = 0; e < per; ++e) {
            const int d = 64 * e + lane;
            s += qv[e] * __builtin_amdgcn_cvt_f32_fp8(kp[((d >> 4) * 16 + i) * 16 + (d & 15)], 0);
            v[e] = __builtin_amdgcn_cvt_f32_fp8(vp[((e * 4 + (i >> 2)) * 16 + (d & 15)) * 16 + ((d >> 4) & 3) * 4 + (i & 3)], 0) * vsc;
        }
        s = wave_sum_fast(s) * ksc;
        if (a.cap > 0.f) s = a.cap * (1.0f - 2.0f / (1.0f + expf(2.0f * (s * a.inv_cap))));
        const float mn = fmaxf(m, s);
        const float al = m == -__builtin_inff() ? 0.f : expf(m - mn), pr = expf(s - mn);
        m = mn;
        l = l * al + pr;
        for (int e = 0; e < per; ++e) o[e] = o[e] * al + pr * v[e];
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    for (int e = 0; e < per; ++e) a.out[t * a.out_stride + head * hd + 64 * e + lane] = (uint16_t)f2bf(o[e] * inv);
}

hipError_t launch_kv8_attention(const Kv8AttnArgs& a, hipStream_t s) {
    const K8Plan p = k8_plan(a);
    const hipError_t e = a.c.hd == 128 ? (p.nt == 1 ? k8_few<128, 1>(a, p, s) : k8_few<128, 2>(a, p, s))
                                       : (p.nt == 1 ? k8_few<64, 1>(a, p, s) : k8_few<64, 2>(a, p, s));
    if (e != hipSuccess || a.max_new * a.G <= 16 * p.nt) return e;
    const int64_t waves = (int64_t)a.T * a.Hq;
    hipLaunchKernelGGL(attn_kv8_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, a, 16 * p.nt);
    return hipGetLastError();
}

}  // namespace mg
