// k_kv8.hip -- the 8-bit paged K/V cache: append with quantisation, and the read back.
//
// A page's 16 positions of one KV head share a scale 2^(b - 127) for K and one for V.  Powers of two:
// multiplying by one changes no mantissa, so a code is the nearest e4m3 value whatever the scale, a
// growing scale moves the codes that stay in the normal range exactly, b is a byte, the largest of the bytes
// that the tokens need is the byte that all of them need, and a value read back is exact in bf16.
//
// Measured (us of a call in a captured graph, hd 128): append of 64 single tokens over 8 KV heads 4.9, read of them 3.3; append of
// 12000 tokens in runs over 4 KV heads 9.1 (37 MB, 4.1 TB/s), read 12.0 (3.1); of 50000 over 8 35 and 70 (307 MB: 8.8,
// partly from the memory-side cache, and 4.4 TB/s; a large copy 4.9).  The read fetches 2.2 times the codes: a wave of four slots takes
// 64 bytes of each 128-byte line of K and touches the lines of V twice where its slots pass a multiple of four, and the
// other part belongs to the next block, on another XCD's L2.
#include <type_traits>

#include "mg_device.h"
#include "mg_kernels.h"

namespace mg {

constexpr int KV8_PAGE = 16;
constexpr int KV8_MIN_BYTE = 16;  // 2^(16 - 127) times the least code, 2^-9, is still normal in bf16

// Tokens of a wave's window: 1 up to KV8_FEW (token, KV head) pairs, 8 up to KV8_SOME, 16 above.  A window of several tokens
// does its runs one after the other (single tokens four at a time), but its waves have work where a run is long: with
// windows of one a run of 16 is one wave's and 15 find nothing to do.  Measured at hd 128, us, windows of 1 / 8 / 16:
// 512 pairs in single tokens 4.9 / 5.3 / 7.7, 1024 5.0 / 5.5 / 7.8, 2048 5.7 / 5.7 / 8.0, 8192 12.5 / 7.4 / 9.3; in runs 2000 pairs
// 6.2 / 5.1 / 7.2, 16000 20 / 6.8 / 7.7, 24000 27 / 8.0 / 8.2, 32000 35 / 9.7 / 8.5, 96000 90 / 18 / 13.
constexpr int KV8_FEW = 1024;
constexpr int KV8_SOME = 24576;

typedef float f32x2_q8 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2_q8 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_q8 __attribute__((ext_vector_type(2)));

// Largest magnitudes of bf16 pairs, as the pair of the two halves' maxima (bits without the sign order as
// magnitudes do, those of infinities and NaN above all others).
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_q8, a), __builtin_bit_cast(u16x2_q8, b)));
}
__device__ __forceinline__ uint32_t mag2(uint32_t pair) { return pair & 0x7fff7fffu; }
// the pair with 0 for what is not finite
__device__ __forceinline__ uint32_t fin2(uint32_t pair) {
    return pair & (((pair & 0x7f80u) != 0x7f80u ? 0xffffu : 0u) | ((pair & 0x7f800000u) != 0x7f800000u ? 0xffff0000u : 0u));
}
// scale byte that a finite magnitude (bf16 bits without the sign) needs: 448 = 1.75 * 2^8
__device__ __forceinline__ int need_byte(uint32_t mag) {
    const int b = (int)(mag >> 7) - 8 + ((mag & 0x7fu) > 0x60u);
    return max(b, KV8_MIN_BYTE);
}
// 2^(127 - b), for b up to 254, whose 2^-127 is below the normal range
__device__ __forceinline__ float inverse(int b) { return __uint_as_float((uint32_t)max((254 - b) << 23, 0x00400000)); }
// four finite bf16 values (two pairs) as codes: inv = 2^(127 - b)
__device__ __forceinline__ uint32_t quant4(uint32_t lo, uint32_t hi, float inv) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(bf_lo(lo) * inv, bf_hi(lo) * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(bf_lo(hi) * inv, bf_hi(hi) * inv, w, true);
}
// NaN codes of those that are not finite
__device__ __forceinline__ uint32_t nan4(uint32_t lo, uint32_t hi) {
    const uint32_t a = mag2(lo), b = mag2(hi);
    return ((a & 0xffffu) >= 0x7f80u ? 0x7fu : 0u) | (a >= 0x7f800000u ? 0x7f00u : 0u) |
           ((b & 0xffffu) >= 0x7f80u ? 0x7f0000u : 0u) | (b >= 0x7f800000u ? 0x7f000000u : 0u);
}
// four bf16 values as codes; ODD: some value of the wave's is not finite, and becomes NaN
template <bool ODD>
__device__ __forceinline__ uint32_t codes4(uint32_t lo, uint32_t hi, float inv) {
    return ODD ? quant4(fin2(lo), fin2(hi), inv) | nan4(lo, hi) : quant4(lo, hi, inv);
}
// Per-lane maxima of K's and V's pairs as one pair over `lanes` lanes: K's in the low half, V's in the high
template <int LANES>
__device__ __forceinline__ uint32_t tops(uint32_t k, uint32_t v) {
    const uint32_t kt = max(k & 0xffffu, k >> 16), vt = max(v & 0xffffu, v >> 16);
    uint32_t t = kt | vt << 16;
#pragma unroll
    for (int x = LANES / 2; x >= 1; x >>= 1) t = max2(t, (uint32_t)__shfl_xor((int)t, x, 64));
    return t;
}
__device__ __forceinline__ bool not_finite(uint32_t t) { return (t & 0xffffu) >= 0x7f80u || t >= 0x7f800000u; }
// four codes of one scale as codes of a larger one (shift = 2^(old - new))
__device__ __forceinline__ uint32_t requant4(uint32_t c, float shift) {
    const f32x2_q8 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a.x * shift, a.y * shift, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b.x * shift, b.y * shift, w, true);
}

// The run of tokens t0 .. on a page: positions [o, end) of the page of slot s0, KV head h0, by one wave.  Lane (g, m)
// holds K's position m, features 64 h + 16 g .., and V's positions 4 g .. 4 g + 3, features 64 h + 16 c + m:
// 16-byte pieces of the page, whose words it writes whole.  V's rows are read eight bytes a lane (features 64 h + 4 m ..),
// and their codes change lanes through the wave's part of LDS.  All that a run may need is requested at once:
// its rows, its scales and, where it begins inside a page, the page.
template <int HD>
struct Kv8Words {
    uint32_t w[4][HD / 64][64][4];  // [wave]: pieces of V
};
// byte j of four words as word j
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    w[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    w[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    w[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}
template <int HD>
__device__ __forceinline__ void append_run(const Kv8& c, int t0, int s0, int o, int end, int h0, int lane,
                                           const uint16_t* __restrict__ k, int64_t ks, const uint16_t* __restrict__ v,
                                           int64_t vs, uint32_t (&words)[HD / 64][64][4]) {
    constexpr int H = HD / 64;
    const int m = lane & 15, g = lane >> 4;
    const size_t ph = ((size_t)(s0 / KV8_PAGE) * c.Hkv + h0) * 2;
    uint8_t* page = c.codes + ph * (size_t)(KV8_PAGE * HD);
    uint4 kx[H][2], old[2][H];
    uint2 vx[H][4];  // [h][i]: position 4 g + i
    const bool mine = m >= o && m < end;
    const uint16_t* kr = k + (int64_t)(t0 + (mine ? m - o : 0)) * ks + (size_t)h0 * HD;
    const uint16_t* vr = v + (int64_t)t0 * vs + (size_t)h0 * HD + 4 * m;
    uint32_t ob = 0;
    if (o) ob = *reinterpret_cast<const uint16_t*>(c.scales + ph);
#pragma unroll
    for (int h = 0; h < H; ++h) {
        kx[h][0] = kx[h][1] = make_uint4(0, 0, 0, 0);
        if (mine) {
            kx[h][0] = *reinterpret_cast<const uint4*>(kr + 64 * h + 16 * g);
            kx[h][1] = *reinterpret_cast<const uint4*>(kr + 64 * h + 16 * g + 8);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * g + i;
            vx[h][i] = make_uint2(0, 0);
            if (t >= o && t < end) vx[h][i] = *reinterpret_cast<const uint2*>(vr + (t - o) * vs + 64 * h);
        }
        old[0][h] = old[1][h] = make_uint4(0, 0, 0, 0);
        if (o) {
            old[0][h] = *reinterpret_cast<const uint4*>(page + h * 1024 + lane * 16);
            old[1][h] = *reinterpret_cast<const uint4*>(page + (H + h) * 1024 + lane * 16);
        }
    }
    auto maxima = [&](auto f) {
        uint32_t mk = 0, mv = 0;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                mk = max2(mk, max2(max2(mag2(f(kx[h][e].x)), mag2(f(kx[h][e].y))), max2(mag2(f(kx[h][e].z)), mag2(f(kx[h][e].w)))));
#pragma unroll
                for (int i = 0; i < 2; ++i) mv = max2(mv, max2(mag2(f(vx[h][2 * e + i].x)), mag2(f(vx[h][2 * e + i].y))));
            }
        return tops<64>(mk, mv);
    };
    uint32_t top = maxima([](uint32_t x) { return x; });
    const bool odd = not_finite(top);
    if (odd) top = maxima([](uint32_t x) { return fin2(x); });
    auto store = [&](auto is_odd) {
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const int was = (int)(side ? ob >> 8 : ob & 0xffu);  // 0: the page starts anew
        const int b = max(was, need_byte(side ? top >> 16 : top & 0xffffu));
        const float inv = inverse(b);
        const float shift = __uint_as_float((uint32_t)max(127 + was - b, 0) << 23);
        // positions of this lane's pieces that the run writes, as a byte mask of a word of V or all of K's piece
        uint32_t keep = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) keep |= 4 * g + i >= o && 4 * g + i < end ? 0u : 0xffu << (8 * i);
        if (side == 0) keep = mine ? 0u : 0xffffffffu;
        const bool store = b != was || keep != 0xffffffffu;  // else none of the piece changes
#pragma unroll
        for (int h = 0; h < H; ++h) {
            uint32_t nw[4], ow[4] = {old[side][h].x, old[side][h].y, old[side][h].z, old[side][h].w};
            if (side) {
#pragma unroll
                for (int i = 0; i < 4; ++i) nw[i] = codes4<decltype(is_odd)::value>(vx[h][i].x, vx[h][i].y, inv);
                transpose4(nw);  // word j: feature 64 h + 4 m + j
#pragma unroll
                for (int j = 0; j < 4; ++j) words[h][g * 16 + 4 * (m & 3) + j][m >> 2] = nw[j];
                __builtin_amdgcn_wave_barrier();
                const uint4 x = *reinterpret_cast<const uint4*>(words[h][lane]);
                nw[0] = x.x;
                nw[1] = x.y;
                nw[2] = x.z;
                nw[3] = x.w;
                __builtin_amdgcn_wave_barrier();
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (!side)
                    nw[q] = codes4<decltype(is_odd)::value>(q & 1 ? kx[h][q >> 1].z : kx[h][q >> 1].x, q & 1 ? kx[h][q >> 1].w : kx[h][q >> 1].y, inv);
                const uint32_t kept = was == 0 ? 0u : b != was ? requant4(ow[q], shift) : ow[q];
                nw[q] = (nw[q] & ~keep) | (kept & keep);
            }
            if (store) *reinterpret_cast<uint4*>(page + (side * H + h) * 1024 + lane * 16) = make_uint4(nw[0], nw[1], nw[2], nw[3]);
        }
        if (lane == 0 && b != was) c.scales[ph + side] = (uint8_t)b;
    }
    };
    if (odd)
        store(std::true_type{});
    else
        store(std::false_type{});
}

// Up to four runs of one token each, 16 lanes a run: position sl of the lane's run (-1: none), its token t, KV head h0.
// A lane holds hd / 16 features of K and of V.  The page itself is only touched where the scale grows, by the whole
// wave, before the token's own bytes are written.
template <int HD>
__device__ __forceinline__ void append_singles(const Kv8& c, int t, int sl, int h0, int lane, const uint16_t* __restrict__ k,
                                               int64_t ks, const uint16_t* __restrict__ v, int64_t vs) {
    constexpr int H = HD / 64, F = HD / 16;
    const int m = lane & 15, o = sl % KV8_PAGE;
    const bool live = sl >= 0;
    const size_t ph = ((size_t)(live ? sl / KV8_PAGE : 0) * c.Hkv + h0) * 2;
    uint8_t* page = c.codes + ph * (size_t)(KV8_PAGE * HD);
    uint32_t x[2][F / 2];
    uint32_t ob = 0;
#pragma unroll
    for (int i = 0; i < F / 2; ++i) x[0][i] = x[1][i] = 0;
    if (live) {
        const uint32_t* kr = reinterpret_cast<const uint32_t*>(k + (int64_t)t * ks + (size_t)h0 * HD) + m * (F / 2);
        const uint32_t* vr = reinterpret_cast<const uint32_t*>(v + (int64_t)t * vs + (size_t)h0 * HD) + m * (F / 2);
#pragma unroll
        for (int i = 0; i < F / 2; ++i) {
            x[0][i] = kr[i];
            x[1][i] = vr[i];
        }
        if (o) ob = *reinterpret_cast<const uint16_t*>(c.scales + ph);
    }
    auto maxima = [&](auto f) {
        uint32_t m[2] = {0, 0};
#pragma unroll
        for (int side = 0; side < 2; ++side)
#pragma unroll
            for (int i = 0; i < F / 2; ++i) m[side] = max2(m[side], mag2(f(x[side][i])));
        return tops<16>(m[0], m[1]);
    };
    uint32_t top = maxima([](uint32_t v) { return v; });
    const bool odd = __any(not_finite(top));
    if (odd) top = maxima([](uint32_t v) { return fin2(v); });
    int b[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const int was = (int)(side ? ob >> 8 : ob & 0xffu);
        b[side] = max(was, need_byte(side ? top >> 16 : top & 0xffffu));
        unsigned long long grows = __ballot(live && b[side] != was && m == 0);
        if (grows) {
            while (grows) {
                const int l0 = __ffsll(grows) - 1;
                grows &= grows - 1;
                const int w0 = __builtin_amdgcn_readlane(was, l0), s0 = __builtin_amdgcn_readlane(sl, l0);
                const float shift = __uint_as_float((uint32_t)max(127 + w0 - __builtin_amdgcn_readlane(b[side], l0), 0) << 23);
                uint4* p = reinterpret_cast<uint4*>(c.codes + (((size_t)(s0 / KV8_PAGE) * c.Hkv + h0) * 2 + side) * (size_t)(KV8_PAGE * HD)) + lane;
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    uint4 q = make_uint4(0, 0, 0, 0);
                    if (w0) {
                        q = p[64 * h];
                        q = make_uint4(requant4(q.x, shift), requant4(q.y, shift), requant4(q.z, shift), requant4(q.w, shift));
                    }
                    p[64 * h] = q;
                }
            }
            // the pages are written before the tokens' bytes, which other lanes write
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        if (live && b[side] != was && m == 0) c.scales[ph + side] = (uint8_t)b[side];
    }
    if (!live) return;
    const float ik = inverse(b[0]), iv = inverse(b[1]);
    uint8_t* kd = page + ((m * F / 16) * 16 + o) * 16 + m * F % 16;
#pragma unroll
    for (int i = 0; i < F / 4; ++i) {
        reinterpret_cast<uint32_t*>(kd)[i] = odd ? codes4<true>(x[0][2 * i], x[0][2 * i + 1], ik) : codes4<false>(x[0][2 * i], x[0][2 * i + 1], ik);
        const uint32_t q = odd ? codes4<true>(x[1][2 * i], x[1][2 * i + 1], iv) : codes4<false>(x[1][2 * i], x[1][2 * i + 1], iv);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int d = m * F + 4 * i + e;
            page[KV8_PAGE * HD + (((d >> 6) * 4 + (o >> 2)) * 16 + (d & 15)) * 16 + ((d >> 4) & 3) * 4 + (o & 3)] = (uint8_t)(q >> (8 * e));
        }
    }
}

// One wave per (window of W tokens, KV head): it does the runs that begin in its window, so one wave alone
// writes a page of a head; with windows of several tokens four runs of one token at a time, the others one
// after the other.
template <int HD, int W>
__global__ __launch_bounds__(256) void kv8_append_kernel(Kv8 c, int n, const uint16_t* __restrict__ k, int64_t ks,
                                                         const uint16_t* __restrict__ v, int64_t vs,
                                                         const int32_t* __restrict__ slots) {
    __shared__ __attribute__((aligned(16))) Kv8Words<HD> sh;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t w = (int64_t)blockIdx.x * 4 + wave;
    const int64_t base = w / c.Hkv * W;
    const int h0 = (int)(w % c.Hkv);
    if (base >= n) return;
    // lane l: the slot of token base - 1 + l, to the end of a run that begins with the window's last token
    const int64_t at = base - 1 + lane;
    const int sl = at >= 0 && at < n && lane <= W + KV8_PAGE - 1 ? slots[at] : -1;
    const bool in = sl >= 0 && sl < (int64_t)c.n_pages * KV8_PAGE;
    const int before = __shfl_up(sl, 1, 64), after = __shfl_down(sl, 1, 64);
    const bool begins = lane >= 1 && lane <= W && in && (sl % KV8_PAGE == 0 || before != sl - 1);
    const bool single = W > 1 && begins && (sl % KV8_PAGE == KV8_PAGE - 1 || after != sl + 1);
    unsigned long long ones = __ballot(single), first = __ballot(begins && !single);
    while (ones) {
        int l0 = 0;
        bool have = false;
#pragma unroll
        for (int r = 0; r < 4; ++r) {  // lane group r takes the r-th run that is left
            if (ones && (lane >> 4) == r) {
                l0 = __ffsll(ones) - 1;
                have = true;
            }
            ones &= ones - 1;
        }
        const int s0 = __shfl(sl, l0, 64);
        append_singles<HD>(c, (int)base - 1 + l0, have ? s0 : -1, h0, lane, k, ks, v, vs);
    }
    while (first) {
        const int l0 = __ffsll(first) - 1;
        first &= first - 1;
        const int s0 = __builtin_amdgcn_readlane(sl, l0), o = s0 % KV8_PAGE, i = lane - l0;
        const unsigned long long run = __ballot(i >= 0 && i < KV8_PAGE - o && sl == s0 + i) >> l0;
        append_run<HD>(c, (int)base - 1 + l0, s0, o, o + __ffsll(~run) - 1, h0, lane, k, ks, v, vs, sh.w[wave]);
    }
}

hipError_t launch_kv8_append(const Kv8& c, int n, const uint16_t* k, int64_t ks, const uint16_t* v, int64_t vs,
                             const int32_t* slots, hipStream_t s) {
    const int64_t pairs = (int64_t)n * c.Hkv;
    const int W = pairs <= KV8_FEW ? 1 : pairs <= KV8_SOME ? 8 : 16;
    const dim3 grid((unsigned)((((int64_t)n + W - 1) / W * c.Hkv + 3) / 4));
    auto f = c.hd == 128 ? (W == 1 ? kv8_append_kernel<128, 1> : W == 8 ? kv8_append_kernel<128, 8> : kv8_append_kernel<128, 16>)
                         : (W == 1 ? kv8_append_kernel<64, 1> : W == 8 ? kv8_append_kernel<64, 8> : kv8_append_kernel<64, 16>);
    hipLaunchKernelGGL(f, grid, dim3(256), 0, s, c, n, k, ks, v, vs, slots);
    return hipGetLastError();
}

// two of a word's codes times 2^(b - 127) (the float f) as a bf16 pair, exact
template <bool HI>
__device__ __forceinline__ uint32_t value2(uint32_t w, float f) {
    return __builtin_bit_cast(uint32_t, (bf16x2_q8)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, HI));
}
// One wave per (four slots of the list, KV head), 16 lanes a slot.  K: lane m has the 16-byte piece of features
// 16 m ..; V: lane m the pieces of features 16 c + m, whose words hold four positions (the four slots of a
// wave mostly), of which it takes its own; the row goes through LDS to be written 16 bytes a lane.
template <int HD>
__global__ __launch_bounds__(256) void kv8_read_kernel(Kv8 c, int n, const int32_t* __restrict__ slots,
                                                       uint16_t* __restrict__ k, int64_t ks, uint16_t* __restrict__ v,
                                                       int64_t vs) {
    constexpr int H = HD / 64;
    __shared__ __attribute__((aligned(16))) uint16_t sh[16][HD + 8];  // a slot's row of V
    const int lane = threadIdx.x & 63, m = lane & 15;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t i = w / c.Hkv * 4 + (lane >> 4);
    const int h0 = (int)(w % c.Hkv);
    if (i >= n) return;
    const int s0 = slots[i];
    if (s0 < 0 || s0 >= (int64_t)c.n_pages * KV8_PAGE) return;
    const int t = s0 % KV8_PAGE;
    const size_t ph = ((size_t)(s0 / KV8_PAGE) * c.Hkv + h0) * 2;
    const uint8_t* page = c.codes + ph * (size_t)(KV8_PAGE * HD);
    const uint32_t sc = *reinterpret_cast<const uint16_t*>(c.scales + ph);
    uint4 kp = make_uint4(0, 0, 0, 0), vp[H];
    if (k && m < HD / 16) kp = *reinterpret_cast<const uint4*>(page + (m * 16 + t) * 16);
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (v) vp[h] = *reinterpret_cast<const uint4*>(page + ((H + h) * 4 + (t >> 2)) * 256 + m * 16);
    if (k && m < HD / 16) {
        const float f = __uint_as_float((sc & 0xffu) << 23);
        const uint32_t q[4] = {kp.x, kp.y, kp.z, kp.w};
        uint32_t o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = e & 1 ? value2<true>(q[e >> 1], f) : value2<false>(q[e >> 1], f);
        uint4* out = reinterpret_cast<uint4*>(k + i * ks + (size_t)h0 * HD + 16 * m);
        out[0] = make_uint4(o[0], o[1], o[2], o[3]);
        out[1] = make_uint4(o[4], o[5], o[6], o[7]);
    }
    if (v) {
        const float f = __uint_as_float((sc >> 8) << 23);
        uint16_t* row = sh[threadIdx.x >> 4];
        const uint32_t pick = (t & 3) * 0x0101u + 0x0400u;  // byte t % 4 of two words
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const uint32_t w = __builtin_amdgcn_perm(vp[h].y, vp[h].x, pick) & 0xffffu | __builtin_amdgcn_perm(vp[h].w, vp[h].z, pick) << 16;
            const uint32_t lo = value2<false>(w, f), hi = value2<true>(w, f);
            row[64 * h + m] = (uint16_t)lo;
            row[64 * h + 16 + m] = (uint16_t)(lo >> 16);
            row[64 * h + 32 + m] = (uint16_t)hi;
            row[64 * h + 48 + m] = (uint16_t)(hi >> 16);
        }
        __builtin_amdgcn_wave_barrier();
        using piece = uint32_t __attribute__((ext_vector_type(HD / 32)));  // the row in 16 pieces
        *reinterpret_cast<piece*>(v + i * vs + (size_t)h0 * HD + HD / 16 * m) = *reinterpret_cast<const piece*>(row + HD / 16 * m);
    }
}

hipError_t launch_kv8_read(const Kv8& c, int n, const int32_t* slots, uint16_t* k, int64_t ks, uint16_t* v, int64_t vs,
                           hipStream_t s) {
    const dim3 grid((unsigned)((((int64_t)n + 3) / 4 * c.Hkv + 3) / 4));
    if (c.hd == 128)
        hipLaunchKernelGGL(kv8_read_kernel<128>, grid, dim3(256), 0, s, c, n, slots, k, ks, v, vs);
    else
        hipLaunchKernelGGL(kv8_read_kernel<64>, grid, dim3(256), 0, s, c, n, slots, k, ks, v, vs);
    return hipGetLastError();
}

}  // namespace mg
