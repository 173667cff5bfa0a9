// k_kv8.hip -- the 8-bit paged K/V cache: append with quantisation, and the read back.
//
// A page's 16 positions of one KV head share a scale 2^(b - 127) for K and one for V.  Powers of two:
// multiplying by one changes no mantissa, so a code is the nearest e4m3 value whatever the scale, a
// growing scale moves the codes that stay in the normal range exactly, b is a byte, the largest of the bytes
// that the tokens need is the byte that all of them need, and a value read back is exact in bf16.
#include "mg_device.h"
#include "mg_kernels.h"

namespace mg {

constexpr int KV8_PAGE = 16;
constexpr int KV8_MIN_BYTE = 16;  // 2^(16 - 127) times the least code, 2^-9, is still normal in bf16

__device__ __forceinline__ size_t k8_off(int t, int d) { return (size_t)((((d >> 4) * 16) + t) * 16 + (d & 15)); }
__device__ __forceinline__ size_t v8_off(int t, int d) {
    return (size_t)((((d >> 6) * 4 + (t >> 2)) * 16 + (d & 15)) * 16 + ((d >> 4) & 3) * 4 + (t & 3));
}

__device__ __forceinline__ bool finite_bf(uint32_t h) { return (h & 0x7f80u) != 0x7f80u; }
// scale byte that a finite magnitude (bf16 bits without the sign) needs: 448 = 1.75 * 2^8
__device__ __forceinline__ int need_byte(uint32_t mag) {
    const int b = (int)(mag >> 7) - 8 + ((mag & 0x7fu) > 0x60u);
    return max(b, KV8_MIN_BYTE);
}
// one bf16 value as a code of scale byte b
__device__ __forceinline__ uint32_t quant(uint32_t h, int b) {
    if (!finite_bf(h)) return 0x7fu;
    const float x = bf2f(h) * __uint_as_float((uint32_t)(254 - b) << 23);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, 0.0f, 0, false) & 0xffu;
}
// a code of one scale as a code of a larger one (shift: 2^(old - new)); no shift: empty
__device__ __forceinline__ uint32_t requant(uint32_t c, float shift) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8((int)c, 0) * shift, 0.0f, 0, false) &
           0xffu;
}

// One wave per (token, KV head); the wave of the first token of a page's run does the run.
__global__ __launch_bounds__(256) void kv8_append_kernel(Kv8 c, int n, const uint16_t* __restrict__ k, int64_t ks,
                                                         const uint16_t* __restrict__ v, int64_t vs,
                                                         const int32_t* __restrict__ slots) {
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t0 = (int)(w / c.Hkv), h = (int)(w % c.Hkv);
    if (t0 >= n) return;
    const int64_t n_slots = (int64_t)c.n_pages * KV8_PAGE;
    const int s0 = slots[t0];
    if (s0 < 0 || s0 >= n_slots) return;
    const int o = s0 % KV8_PAGE;
    if (o > 0 && t0 > 0 && slots[t0 - 1] == s0 - 1) return;
    int cnt = 1;
    while (o + cnt < KV8_PAGE && t0 + cnt < n && slots[t0 + cnt] == s0 + cnt) ++cnt;
    const int hd = c.hd, pg = s0 / KV8_PAGE;
    for (int side = 0; side < 2; ++side) {
        const uint16_t* x = (side ? v + (int64_t)t0 * vs : k + (int64_t)t0 * ks) + h * hd;
        const int64_t xs = side ? vs : ks;
        const size_t ph = ((size_t)pg * c.Hkv + h) * 2 + side;
        uint8_t* page = c.codes + ph * (size_t)(KV8_PAGE * hd);
        uint32_t top = 0;
        for (int i = 0; i < cnt; ++i)
            for (int d = lane; d < hd; d += 64) {
                const uint32_t e = x[i * xs + d];
                if (finite_bf(e)) top = max(top, e & 0x7fffu);
            }
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m, 64));
        const int old = o == 0 ? 0 : c.scales[ph];
        const int b = max(old, need_byte(top));
        if (b != old) {
            const float shift = __uint_as_float((uint32_t)max(127 + old - b, 0) << 23);
            for (int t = 0; t < KV8_PAGE; ++t) {
                if (t >= o && t < o + cnt) continue;
                for (int d = lane; d < hd; d += 64) {
                    uint8_t* p = page + (side ? v8_off(t, d) : k8_off(t, d));
                    *p = old ? (uint8_t)requant(*p, shift) : 0;
                }
            }
            if (lane == 0) c.scales[ph] = (uint8_t)b;
        }
        for (int i = 0; i < cnt; ++i)
            for (int d = lane; d < hd; d += 64)
                page[side ? v8_off(o + i, d) : k8_off(o + i, d)] = (uint8_t)quant(x[i * xs + d], b);
    }
}

hipError_t launch_kv8_append(const Kv8& c, int n, const uint16_t* k, int64_t ks, const uint16_t* v, int64_t vs,
                             const int32_t* slots, hipStream_t s) {
    const int64_t waves = (int64_t)n * c.Hkv;
    hipLaunchKernelGGL(kv8_append_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, c, n, k, ks, v, vs,
                       slots);
    return hipGetLastError();
}

// One wave per (slot, KV head).
__global__ __launch_bounds__(256) void kv8_read_kernel(Kv8 c, int n, const int32_t* __restrict__ slots,
                                                       uint16_t* __restrict__ k, int64_t ks, uint16_t* __restrict__ v,
                                                       int64_t vs) {
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t i = w / c.Hkv;
    const int h = (int)(w % c.Hkv);
    if (i >= n) return;
    const int s0 = slots[i];
    if (s0 < 0 || s0 >= (int64_t)c.n_pages * KV8_PAGE) return;
    const int t = s0 % KV8_PAGE, hd = c.hd;
    for (int side = 0; side < 2; ++side) {
        uint16_t* out = side ? v : k;
        if (!out) continue;
        out += i * (side ? vs : ks) + h * hd;
        const size_t ph = ((size_t)(s0 / KV8_PAGE) * c.Hkv + h) * 2 + side;
        const uint8_t* page = c.codes + ph * (size_t)(KV8_PAGE * hd);
        const float scale = __uint_as_float((uint32_t)c.scales[ph] << 23);
        for (int d = lane; d < hd; d += 64) {
            const uint32_t e = page[side ? v8_off(t, d) : k8_off(t, d)];
            out[d] = (uint16_t)f2bf(__builtin_amdgcn_cvt_f32_fp8((int)e, 0) * scale);
        }
    }
}

hipError_t launch_kv8_read(const Kv8& c, int n, const int32_t* slots, uint16_t* k, int64_t ks, uint16_t* v, int64_t vs,
                           hipStream_t s) {
    const int64_t waves = (int64_t)n * c.Hkv;
    hipLaunchKernelGGL(kv8_read_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, c, n, slots, k, ks, v, vs);
    return hipGetLastError();
}

}  // namespace mg
