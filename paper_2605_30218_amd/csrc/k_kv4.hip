// k_kv4.hip -- rotation and append of a batch's new tokens into the 4-bit paged K/V cache, and the read of its values.
//
// A pair (i, i + hd/2) of a head at position p turns by the angle of table row p: (a c - b s, b c + a s), products and sums
// rounded to fp32 each, the result to bf16, as the decode path's own rotation.  A block of values (32 features of a key, a whole
// value) becomes e2m1 codes under the least power of two whose sevenfold holds its largest magnitude: dividing by it is exact, so a
// code is the nearest one whatever the scale, and nothing written before is rounded again.
//
// Many tokens are bound by bytes: 12000 of 28 query heads over 4 of 128 take 37.6 us, 203 MB at 5.4 TB/s (as a copy of 200 MiB), the read
// of them 8.1 us; few by the chain of slot, row, maximum, code: 64 tokens of 32 heads over 8 4.5 us, their read 2.9, a launch that does nothing 1.6.
#include "mg_device.h"
#include "mg_kernels.h"

namespace mg {
namespace {

typedef uint32_t u32x4_k4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_k4 __attribute__((ext_vector_type(2)));

constexpr int K4_THREADS = 256;
constexpr int K4_NAN = 255;  // scale byte of a block that holds a value that is not finite

// the scale byte of a block from its largest bf16 magnitude's bits: 7 * 2^(b - 127) >= that magnitude
__device__ __forceinline__ int k4_scale_byte(uint32_t top) {
    const int b = (int)(top >> 7) - 2 + ((top & 0x7fu) > 0x60u ? 1 : 0);
    return top >= 0x7f80u ? K4_NAN : max(b, 16);
}
// 2^(127 - b): what takes a block's values to its codes' range (0 for a block that is not finite)
__device__ __forceinline__ float k4_unit(int b) { return __uint_as_float(b == K4_NAN ? 0u : (uint32_t)(254 - b) << 23); }
// two values in a code's range as codes, the first in the low nibble (0 where they are not finite)
template <int BYTE>
__device__ __forceinline__ uint32_t k4_codes(uint32_t old, float lo, float hi) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, lo, hi, 1.0f, BYTE);
}
// the larger magnitude of each half of two words of bf16 pairs
__device__ __forceinline__ uint32_t k4_top2(uint32_t a, uint32_t b) {
    a &= 0x7fff7fffu;
    b &= 0x7fff7fffu;
    return max(a & 0xffffu, b & 0xffffu) | (max(a >> 16, b >> 16) << 16);
}
__device__ __forceinline__ uint32_t k4_top(const uint32_t (&w)[4]) {
    const uint32_t m = k4_top2(k4_top2(w[0], w[1]), k4_top2(w[2], w[3]));
    return max(m & 0xffffu, m >> 16);
}

// eight values of a head as codes of the block that four neighbouring lanes share, into the cache
__device__ __forceinline__ void k4_put_k(const uint32_t (&w)[4], uint8_t* codes, uint8_t* scales, int block, int t) {
    const int part = threadIdx.x & 3;
    uint32_t top = k4_top(w);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    const int b = k4_scale_byte(top);
    const float u = k4_unit(b);
    uint32_t c = 0;
    if (b != K4_NAN) {
        c = k4_codes<0>(c, bf_lo(w[0]) * u, bf_hi(w[0]) * u);
        c = k4_codes<1>(c, bf_lo(w[1]) * u, bf_hi(w[1]) * u);
        c = k4_codes<2>(c, bf_lo(w[2]) * u, bf_hi(w[2]) * u);
        c = k4_codes<3>(c, bf_lo(w[3]) * u, bf_hi(w[3]) * u);
    }
    const int at = block * 16 + t;
    *reinterpret_cast<uint32_t*>(codes + at * 16 + part * 4) = c;
    if (part == 0) scales[at] = (uint8_t)b;
}

// a token's page and position, or page -1 where nothing is stored for it
struct K4At {
    int page, t;
};
__device__ __forceinline__ K4At k4_at(const Kv4AppendArgs& a, int slot, int pos) {
    const bool ok = slot >= 0 && (slot >> 4) < a.c.n_pages && pos >= 0;
    return K4At{ok ? slot >> 4 : -1, slot & 15};
}

// Queries and keys: HD / 16 lanes a head, each with eight pairs (i, i + HD / 2) of it; a lane takes U heads of a token and reads
// the angles once for them.
template <int HD, int U>
__device__ __forceinline__ void k4_rotate(const Kv4AppendArgs& a, int block) {
    constexpr int LPH = HD / 16, H2 = HD / 2;
    const int heads = a.Hq + a.c.Hkv, groups = (heads + U - 1) / U;
    const int64_t task = (int64_t)block * K4_THREADS + threadIdx.x;
    const int unit = (int)(task / LPH), at = (int)(task % LPH) * 8;
    const int tok = unit / groups, h0 = unit % groups;
    if (tok >= a.n) return;
    uint4 lo[U], hi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u * groups;
        if (h < heads) {
            const uint16_t* p = (h < a.Hq ? a.q + tok * a.q_stride + h * HD : a.k + tok * a.k_stride + (h - a.Hq) * HD) + at;
            lo[u] = *reinterpret_cast<const uint4*>(p);
            hi[u] = *reinterpret_cast<const uint4*>(p + H2);
        }
    }
    float cs[16];
    const int slot = a.slots[tok], pos = a.positions ? a.positions[tok] : 0;
    if (pos < 0) return;
    if (a.positions) {
        if (pos < a.n_positions) {
            const float* r = a.rope + (int64_t)pos * HD + 2 * at;
#pragma unroll
            for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(cs + i) = *reinterpret_cast<const float4*>(r + i);
        } else {  // the table has no angle for it
#pragma unroll
            for (int i = 0; i < 16; ++i) cs[i] = __builtin_nanf("");
        }
    }
    const K4At where = k4_at(a, slot, pos);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u * groups;
        if (h >= heads) break;
        uint32_t x[4] = {lo[u].x, lo[u].y, lo[u].z, lo[u].w}, y[4] = {hi[u].x, hi[u].y, hi[u].z, hi[u].w};
        if (a.positions) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a0 = bf_lo(x[i]), a1 = bf_hi(x[i]), b0 = bf_lo(y[i]), b1 = bf_hi(y[i]);
                const float c0 = cs[4 * i], s0 = cs[4 * i + 1], c1 = cs[4 * i + 2], s1 = cs[4 * i + 3];
                x[i] = pack_bf2(a0 * c0 - b0 * s0, a1 * c1 - b1 * s1);
                y[i] = pack_bf2(b0 * c0 + a0 * s0, b1 * c1 + a1 * s1);
            }
        }
        if (h < a.Hq) {
            uint16_t* o = a.q_out + tok * a.q_out_stride + h * HD + at;
            *reinterpret_cast<uint4*>(o) = make_uint4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<uint4*>(o + H2) = make_uint4(y[0], y[1], y[2], y[3]);
        } else if (where.page >= 0) {
            const size_t ph = (size_t)where.page * a.c.Hkv + (h - a.Hq);
            uint8_t* codes = a.c.codes + ph * (16 * HD);
            uint8_t* scales = a.c.scales + ph * (HD / 2 + 16);
            k4_put_k(x, codes, scales, at / 32, where.t);
            k4_put_k(y, codes, scales, (at + H2) / 32, where.t);
        }
    }
}

// Values: two positions share a byte, and four stand in 16 (HD 128) or 8 bytes of a lane.  Tokens that stand together in the call and in four aligned
// positions of a page (up to four of a row, as a batch plan lists them) are written by the first of them: by plain stores where they are all
// four, else by changing their own bits alone, as other tokens of the call may change the others at the same time.  Of two tokens with the same slot within
// four the earlier one is left out.  16 lanes a head, lane m with features 16 c + m.  (The neighbours' slots by a lane each and all that follows from them in
// scalar registers: 64 tokens 4.5 us, with the loads and comparisons in every lane 5.4; plain stores where no other token can be near: no gain.)
template <int HD>
__device__ __forceinline__ void k4_values(const Kv4AppendArgs& a, int block) {
    constexpr int C = HD / 16;
    const int m = threadIdx.x & 15;
    const int64_t task = ((int64_t)block * K4_THREADS + threadIdx.x) >> 4;
    const int groups = (a.c.Hkv + 3) / 4;  // (a wave's four heads are one token's)
    const int tok = __builtin_amdgcn_readfirstlane((int)(task / 4 / groups)), h = (int)(task / 4 % groups * 4 + task % 4);
    if (tok >= a.n || h >= a.c.Hkv) return;
    int near[8];  // slots of the tokens from tok - 1 to tok + 6 (-1: nothing is stored), a lane each
    {
        const int o = tok - 1 + (int)(threadIdx.x & 7), in = min(max(o, 0), a.n - 1);
        const int slot = a.slots[in], pos = a.positions ? a.positions[in] : 0;
        const int own = k4_at(a, slot, o == in ? pos : -1).page < 0 ? -1 : slot;
#pragma unroll
        for (int i = 0; i < 8; ++i) near[i] = __builtin_amdgcn_readlane(own, i);
    }
    // whether neighbour i is of the four positions of tok's, and none of the three behind it has its slot
    const auto here = [&](int i) {
        return near[i] >> 2 == near[1] >> 2 && near[i] != near[i + 1] && near[i] != near[i + 2] && near[i] != near[i + 3];
    };
    if (near[1] < 0 || !here(1) || here(0)) return;
    const K4At at{near[1] >> 4, near[1] & 15};
    int src[4] = {-1, -1, -1, -1};  // the token at each of the four positions
    bool run = true;
#pragma unroll
    for (int i = 1; i < 5; ++i) {
        run = run && here(i);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (run && (near[i] & 3) == j) src[j] = tok + i - 1;
    }
    uint32_t keep = 0;  // the nibbles of the positions that have none
#pragma unroll
    for (int i = 0; i < 4; ++i) keep |= src[i] < 0 ? 15u << (4 * i) : 0u;
    keep |= keep << 16;
    const size_t ph = (size_t)at.page * a.c.Hkv + h;
    uint8_t* codes = a.c.codes + ph * (16 * HD) + 8 * HD + ((at.t >> 2) * 16 + m) * (HD / 8);
    uint8_t* scales = a.c.scales + ph * (HD / 2 + 16) + HD / 2 + (at.t & ~3);
    uint32_t w[C / 2];  // tiles 2 i and 2 i + 1, four positions each
    if (keep) {
#pragma unroll
        for (int i = 0; i < C / 2; ++i) w[i] = reinterpret_cast<const uint32_t*>(codes)[i];
    }
    uint16_t x[4][C];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint16_t* p = a.v + (int64_t)max(src[i], tok) * a.v_stride + h * HD + m;
#pragma unroll
        for (int c = 0; c < C; ++c) x[i][c] = src[i] >= 0 ? p[16 * c] : (uint16_t)0;
    }
    float u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) top = max(top, (uint32_t)x[i][c] & 0x7fffu);
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
        const int b = k4_scale_byte(top);
        u[i] = k4_unit(b);
        if (m == 0 && src[i] >= 0) scales[i] = (uint8_t)b;
    }
#pragma unroll
    for (int i = 0; i < C / 2; ++i) {
        uint32_t n = 0;
        // (infinity times 0 is NaN and becomes some code: its byte says that the value is none)
        n = k4_codes<0>(n, bf2f(x[0][2 * i]) * u[0], bf2f(x[1][2 * i]) * u[1]);
        n = k4_codes<1>(n, bf2f(x[2][2 * i]) * u[2], bf2f(x[3][2 * i]) * u[3]);
        n = k4_codes<2>(n, bf2f(x[0][2 * i + 1]) * u[0], bf2f(x[1][2 * i + 1]) * u[1]);
        n = k4_codes<3>(n, bf2f(x[2][2 * i + 1]) * u[2], bf2f(x[3][2 * i + 1]) * u[3]);
        w[i] = keep ? (n ^ w[i]) & ~keep : n;  // (what changes)
    }
    if (keep) {
#pragma unroll
        for (int i = 0; i < C / 2; i += 2)
            atomicXor(reinterpret_cast<unsigned long long*>(codes) + i / 2, w[i] | (unsigned long long)w[i + 1] << 32);
    } else if constexpr (C == 8) {
        *reinterpret_cast<uint4*>(codes) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        *reinterpret_cast<uint2*>(codes) = make_uint2(w[0], w[1]);
    }
}

template <int HD, int U>
__global__ __launch_bounds__(K4_THREADS) void kv4_append_kernel(Kv4AppendArgs a, int rotate_blocks) {
    if ((int)blockIdx.x < rotate_blocks)
        k4_rotate<HD, U>(a, blockIdx.x);
    else
        k4_values<HD>(a, blockIdx.x - rotate_blocks);
}

// Read: HD / 8 lanes a slot of a head, each with eight features.  (V by eight loads of a byte a lane: 12000 slots of 4 heads 9.4 us instead of 8.2.)
template <int HD>
__global__ __launch_bounds__(K4_THREADS) void kv4_read_kernel(Kv8 c, int n, const int32_t* __restrict__ slots, uint16_t* k,
                                                              int64_t ks, uint16_t* v, int64_t vs) {
    constexpr int L = HD / 8;
    __shared__ uint32_t all[K4_THREADS];
    const int64_t task = (int64_t)blockIdx.x * K4_THREADS + threadIdx.x;
    const int lane = (int)(task % L), h = (int)(task / L % c.Hkv);
    const int64_t i = task / L / c.Hkv;
    if (i >= n) return;
    const int s = slots[i], page = s >> 4, t = s & 15;
    if (s < 0 || page >= c.n_pages) return;
    const size_t ph = (size_t)page * c.Hkv + h;
    const uint8_t* codes = c.codes + ph * (16 * HD);
    const uint8_t* scales = c.scales + ph * (HD / 2 + 16);
    auto put = [&](uint32_t w, int b, uint16_t* p) {  // eight codes, the first in the lowest nibble
        const float f = __uint_as_float((uint32_t)max(b, 1) << 23);
        uint4 o;
        o.x = __builtin_bit_cast(uint32_t, (bf16x2_k4)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 0));
        o.y = __builtin_bit_cast(uint32_t, (bf16x2_k4)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 1));
        o.z = __builtin_bit_cast(uint32_t, (bf16x2_k4)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 2));
        o.w = __builtin_bit_cast(uint32_t, (bf16x2_k4)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 3));
        if (b == K4_NAN) o = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
        *reinterpret_cast<uint4*>(p) = o;
    };
    if (k) {
        const int at = lane / 4 * 16 + t;
        put(*reinterpret_cast<const uint32_t*>(codes + at * 16 + lane % 4 * 4), scales[at], k + i * ks + h * HD + 8 * lane);
    }
    if (v) {
        // A position's codes lie at every second byte or so of its four positions': a lane loads what it has of 16 bytes (HD 128: its
        // feature m of all tiles, HD 64: two), keeps the nibbles of its position, and takes the other lanes' by way of LDS.
        const u32x4_k4 x = *reinterpret_cast<const u32x4_k4*>(codes + 8 * HD + (t >> 2) * (2 * HD) + lane * 16);
        uint32_t own = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t y = x[j] >> (4 * (t & 3)) & 0x000f000fu;
            own |= ((y | y >> 12) & 0xffu) << (8 * j);
        }
        all[threadIdx.x] = own;
        // (the lanes of a slot are of one wave, whose LDS accesses keep their order)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        uint32_t w = 0;
#pragma unroll
        for (int m = 0; m < 8; ++m) {  // features 8 lane .. of tile lane / 2
            const uint32_t o = all[threadIdx.x - lane + (HD == 128 ? lane % 2 * 8 + m : lane % 2 * 4 + m / 2)];
            w |= (o >> (lane / 2 * 4 + (HD == 128 ? 0 : m % 2 * 16)) & 15u) << (4 * m);
        }
        put(w, scales[HD / 2 + t], v + i * vs + h * HD + 8 * lane);
    }
}

template <int HD>
void append(const Kv4AppendArgs& a, hipStream_t s) {
    const int heads = a.Hq + a.c.Hkv;
    // (heads of a lane: with 1, 2, 4, 8 of them 64 tokens of 40 heads take 4.4, 4.4, 5.8, 9.0 us, 12000 of 32 39.5, 37.6, 37.8, 38.7, 12000 of 40
    // 56, 54, 53, 55)
    constexpr int U = 2;
    const int64_t lanes = (int64_t)a.n * ((heads + U - 1) / U) * (HD / 16);
    const int64_t rot = (lanes + K4_THREADS - 1) / K4_THREADS;
    const int64_t val = ((int64_t)a.n * ((a.c.Hkv + 3) / 4) * 64 + K4_THREADS - 1) / K4_THREADS;
    hipLaunchKernelGGL((kv4_append_kernel<HD, U>), dim3((unsigned)(rot + val)), dim3(K4_THREADS), 0, s, a, (int)rot);
}

}  // namespace

hipError_t launch_kv4_append(const Kv4AppendArgs& a, hipStream_t s) {
    if (a.c.hd == 128)
        append<128>(a, s);
    else
        append<64>(a, s);
    return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv8& c, int n, const int32_t* slots, uint16_t* k, int64_t ks, uint16_t* v, int64_t vs,
                           hipStream_t s) {
    const int64_t blocks = ((int64_t)n * c.Hkv * (c.hd / 8) + K4_THREADS - 1) / K4_THREADS;
    auto f = c.hd == 128 ? kv4_read_kernel<128> : kv4_read_kernel<64>;
    hipLaunchKernelGGL(f, dim3((unsigned)blocks), dim3(K4_THREADS), 0, s, c, n, slots, k, ks, v, vs);
    return hipGetLastError();
}

}  // namespace mg
