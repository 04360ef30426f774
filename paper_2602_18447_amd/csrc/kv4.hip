// The paged cache in 4 bits: append of rotated keys and values, its rows as values, attention over it.  Page format:
// confspec_int4.h.
#include "kernels.h"
#include <algorithm>

namespace cs {

namespace {

__device__ __forceinline__ float bf16_f32(bf16 v) { return __bfloat162float(v); }

// Trace of packed token t: the largest b with cu[b] <= t.
__device__ __forceinline__ int trace_of(const int32_t *cu, int B, int t) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cu[mid] <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}
// Page of cache row `row` of trace b and head h, clamped into the cache.
__device__ __forceinline__ uint8_t *page_of(const Kv4Batch &b, int trace, int row, int h) {
    const int j = min(max(row >> 4, 0), b.max_blocks - 1);
    const int blk = min(max(b.table[(size_t)trace * b.max_blocks + j], 0), b.n_blocks - 1);
    return b.pages + ((size_t)blk * b.Hkv + h) * KV4_PAGE;
}
// Byte offset of the key word that has element d (a multiple of 8) of token t; the value word likewise.
__device__ __forceinline__ int k_word(int t, int d) { return (((((d & 31) >> 3) * 16 + t) * 4) + (d >> 5)) * 4; }
__device__ __forceinline__ int v_word(int t, int d) { return KV4_V + (((t >> 2) * 16 + (d >> 3)) * 4 + (t & 3)) * 4; }
__device__ __forceinline__ int k_shift(int e) { return 4 * ((e >> 1) + 4 * (e & 1)); }

// cos / sin of x >= 0 in 64 bits: reduction by multiples of pi / 2 held in two terms (Cody and Waite), then the Taylor
// series, whose first dropped terms at pi / 4 are below 2^-54.
__device__ __forceinline__ void sincos64(double x, double &s, double &c) {
    const double k = rint(x * 0.63661977236758134308);
    double r = fma(-k, 1.57079632679489661923, x);
    r = fma(-k, 6.12323399573676588613e-17, r);
    const double z = r * r;
    double p = 1.0 / 355687428096000.0;                  // 1 / 17!
    p = fma(p, z, -1.0 / 1307674368000.0);
    p = fma(p, z, 1.0 / 6227020800.0);
    p = fma(p, z, -1.0 / 39916800.0);
    p = fma(p, z, 1.0 / 362880.0);
    p = fma(p, z, -1.0 / 5040.0);
    p = fma(p, z, 1.0 / 120.0);
    p = fma(p, z, -1.0 / 6.0);
    const double sn = fma(r * z, p, r);
    double q = 1.0 / 20922789888000.0;                   // 1 / 16!
    q = fma(q, z, -1.0 / 87178291200.0);
    q = fma(q, z, 1.0 / 479001600.0);
    q = fma(q, z, -1.0 / 3628800.0);
    q = fma(q, z, 1.0 / 40320.0);
    q = fma(q, z, -1.0 / 720.0);
    q = fma(q, z, 1.0 / 24.0);
    q = fma(q, z, -0.5);
    const double cn = fma(q, z, 1.0);
    const int quadrant = (int)((long long)k & 3);
    const double a = quadrant & 1 ? cn : sn, b = quadrant & 1 ? sn : cn;
    s = quadrant & 2 ? -a : a;
    c = (quadrant == 1 || quadrant == 2) ? -b : b;
}

// One workgroup per token, a wavefront per head in turn; lane i has elements i and i + 64.
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4Append a) {
    const Kv4Batch &b = a.b;
    const int t = blockIdx.x, lane = threadIdx.x & 63;
    const int trace = trace_of(b.cu, b.B, t);
    const int i = min(max(t - b.cu[trace], 0), b.T - 1), L = max(b.plens[trace], 0), row = L + i;
    const bool store = (!a.n_append || i < a.n_append[trace]) && row >= 0 && row < b.max_blocks * 16;
    double sn, cn;
    sincos64((double)row * a.inv_freq[lane], sn, cn);
    for (int h = threadIdx.x >> 6; h < a.Hq + 2 * b.Hkv; h += 4) {
        const float *src = a.qkv + (size_t)t * a.stride + (size_t)h * 128;
        float lo = src[lane], hi = src[lane + 64];
        if (h < a.Hq + b.Hkv) {
            const double x = lo, y = hi;
            lo = (float)(x * cn - y * sn);
            hi = (float)(y * cn + x * sn);
        }
        const bf16 l16 = __float2bfloat16(lo), h16 = __float2bfloat16(hi);
        const bool is_k = h >= a.Hq && h < a.Hq + b.Hkv;
        const int hk = is_k ? h - a.Hq : h - a.Hq - b.Hkv;
        bf16 *dst = h < a.Hq ? a.q + ((size_t)t * a.Hq + h) * 128 : (is_k ? a.k : a.v) + ((size_t)t * b.Hkv + hk) * 128;
        dst[lane] = l16;
        dst[lane + 64] = h16;
        if (h < a.Hq || !store) continue;
        // min and max of the row, its pair (s, z), the codes
        const float x0 = __builtin_amdgcn_fmed3f(bf16_f32(l16), -65504.f, 65504.f), x1 = __builtin_amdgcn_fmed3f(bf16_f32(h16), -65504.f, 65504.f);
        float mn = fminf(x0, x1), mx = fmaxf(x0, x1);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) { mn = fminf(mn, __shfl_xor(mn, o, 64)); mx = fmaxf(mx, __shfl_xor(mx, o, 64)); }
        const __half zh = __float2half_rn(mn + 0.f);            // (never -0)
        const float z = __half2float(zh);
        const __half sh = __float2half_rn((float)(((double)mx - (double)z) / 15.0));
        const float s = __half2float(sh);
        const float c0 = s > 0.f ? fminf(fmaxf(rintf((x0 - z) / s), 0.f), 15.f) : 0.f;
        const float c1 = s > 0.f ? fminf(fmaxf(rintf((x1 - z) / s), 0.f), 15.f) : 0.f;
        const int e = lane & 7, sft = is_k ? k_shift(e) : 4 * e;
        unsigned w0 = (unsigned)c0 << sft, w1 = (unsigned)c1 << sft;
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) { w0 |= __shfl_xor((int)w0, o, 64); w1 |= __shfl_xor((int)w1, o, 64); }
        uint8_t *page = page_of(b, trace, row, hk);
        const int slot = row & 15;
        if (e == 0) {
            *(unsigned *)(page + (is_k ? k_word(slot, lane) : v_word(slot, lane))) = w0;
            *(unsigned *)(page + (is_k ? k_word(slot, lane + 64) : v_word(slot, lane + 64))) = w1;
        }
        if (lane == 0)
            *(unsigned *)(page + (is_k ? KV4_KP : KV4_VP) + slot * 4) = (unsigned)__half_as_ushort(sh) | (unsigned)__half_as_ushort(zh) << 16;
    }
}

__device__ __forceinline__ float param_s(unsigned p) { return __half2float(__ushort_as_half((unsigned short)(p & 0xffff))); }
__device__ __forceinline__ float param_z(unsigned p) { return __half2float(__ushort_as_half((unsigned short)(p >> 16))); }

// One workgroup per token; a thread has 8 elements (one word) of a key or value row.
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Batch b, float *__restrict__ k, float *__restrict__ v) {
    const int t = blockIdx.x;
    const int trace = trace_of(b.cu, b.B, t);
    const int row = max(b.plens[trace], 0) + min(max(t - b.cu[trace], 0), b.T - 1), slot = row & 15;
    for (int j = threadIdx.x; j < b.Hkv * 32; j += 256) {
        const int h = j >> 5, is_v = (j >> 4) & 1, d = (j & 15) * 8;
        const uint8_t *page = page_of(b, trace, row, h);
        const unsigned w = *(const unsigned *)(page + (is_v ? v_word(slot, d) : k_word(slot, d)));
        const unsigned p = *(const unsigned *)(page + (is_v ? KV4_VP : KV4_KP) + slot * 4);
        float *dst = (is_v ? v : k) + ((size_t)t * b.Hkv + h) * 128 + d;
#pragma unroll
        for (int e = 0; e < 8; ++e) dst[e] = fmaf(param_s(p), (float)((w >> (is_v ? 4 * e : k_shift(e))) & 15), param_z(p));
    }
}

// One wavefront per (token, q head); 64 keys a round, a lane per key for the scores and per two elements for the sums.
__global__ __launch_bounds__(64) void kv4_attn_kernel(Kv4Attn a) {
    const Kv4Batch &b = a.b;
    __shared__ float sq[128], sp[64];
    const int lane = threadIdx.x, t = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, hk = h / (a.Hq / b.Hkv);
    const int trace = trace_of(b.cu, b.B, t), t0 = b.cu[trace];
    const int L = min(max(b.plens[trace], 0), b.max_blocks * 16), n = L + min(max(t - t0, 0), b.T - 1) + 1;
    const bf16 *q = a.q + ((size_t)t * a.Hq + h) * 128;
    sq[lane] = bf16_f32(q[lane]) * 0.08838834764831845f;
    sq[lane + 64] = bf16_f32(q[lane + 64]) * 0.08838834764831845f;
    __syncthreads();
    float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
    for (int j0 = 0; j0 < n; j0 += 64) {
        const int j = j0 + lane;
        float s = -INFINITY;
        if (j < n) {
            s = 0.f;
            if (j < L) {
                const uint8_t *page = page_of(b, trace, j, hk);
                const unsigned p = *(const unsigned *)(page + KV4_KP + (j & 15) * 4);
                float sum = 0.f;
                for (int d = 0; d < 128; d += 8) {
                    const unsigned w = *(const unsigned *)(page + k_word(j & 15, d));
#pragma unroll
                    for (int e = 0; e < 8; ++e) { s += sq[d + e] * (float)((w >> k_shift(e)) & 15); sum += sq[d + e]; }
                }
                s = param_s(p) * s + param_z(p) * sum;
            } else {
                const bf16 *k = a.k + ((size_t)(t0 + j - L) * b.Hkv + hk) * 128;
                for (int d = 0; d < 128; ++d) s += sq[d] * bf16_f32(k[d]);
            }
        }
        float mx = s;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        const float mn = fmaxf(m, mx), keep = expf(m - mn);
        m = mn;
        sp[lane] = expf(s - m);
        __syncthreads();
        o0 *= keep; o1 *= keep; l *= keep;
        for (int i = 0; i < min(64, n - j0); ++i) {
            const int jj = j0 + i;
            const float p = sp[i];
            l += p;
            if (jj < L) {
                const uint8_t *page = page_of(b, trace, jj, hk);
                const unsigned pr = *(const unsigned *)(page + KV4_VP + (jj & 15) * 4);
                const unsigned w = *(const unsigned *)(page + v_word(jj & 15, 2 * lane & ~7));
                const int sh = 4 * (2 * lane & 7);
                o0 += p * fmaf(param_s(pr), (float)((w >> sh) & 15), param_z(pr));
                o1 += p * fmaf(param_s(pr), (float)((w >> (sh + 4)) & 15), param_z(pr));
            } else {
                const bf16 *v = a.v + ((size_t)(t0 + jj - L) * b.Hkv + hk) * 128;
                o0 += p * bf16_f32(v[2 * lane]);
                o1 += p * bf16_f32(v[2 * lane + 1]);
            }
        }
        __syncthreads();
    }
    bf16 *out = a.out + ((size_t)t * a.Hq + h) * 128;
    out[2 * lane] = __float2bfloat16(o0 / l);
    out[2 * lane + 1] = __float2bfloat16(o1 / l);
}

}  // namespace

hipError_t launch_kv4_append(const Kv4Append &a, hipStream_t s) {
    kv4_append_kernel<<<a.b.T, 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4Batch &b, float *k, float *v, hipStream_t s) {
    kv4_read_kernel<<<b.T, 256, 0, s>>>(b, k, v);
    return hipGetLastError();
}

size_t kv4_attn_scratch(const int32_t *, const int32_t *, int, int, int) { return 0; }

hipError_t launch_kv4_attn(const Kv4Attn &a, const int32_t *, const int32_t *, void *, hipStream_t s) {
    kv4_attn_kernel<<<a.b.T * a.Hq, 64, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cs
