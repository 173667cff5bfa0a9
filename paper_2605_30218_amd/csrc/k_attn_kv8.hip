// k_attn_kv8.hip -- attention of a batch's new tokens over the 8-bit paged K/V cache.
//
// One wave per (token, query head): a pass over the positions that the token sees with the running
// maximum, sum and output of the softmax, a lane holding hd / 64 features.
#include "mg_device.h"
#include "mg_kernels.h"

namespace mg {

__global__ __launch_bounds__(256) void attn_kv8_kernel(Kv8AttnArgs a) {
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

size_t kv8_attention_ws_bytes(const Kv8AttnArgs&) { return 0; }

hipError_t launch_kv8_attention(const Kv8AttnArgs& a, hipStream_t s) {
    const int64_t waves = (int64_t)a.T * a.Hq;
    hipLaunchKernelGGL(attn_kv8_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace mg
