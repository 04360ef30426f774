// Products of up to 128 rows with 4-bit weights.  Record format: confspec_int4.h, kernels.h.
#include "kernels.h"

namespace cs {

namespace {

// Row of the matrix that is row m of the 16 of tile nt.  A gate/up matrix has gate f, f + 1 and up f, f + 1 in turn, so
// that the four rows a lane gets from a matrix instruction are two finished pairs.
__device__ __forceinline__ int w4_source_row(int nt, int m, int N, int gate_up) {
    if (!gate_up) return nt * 16 + m;
    const int f = nt * 8 + (m >> 2) * 2 + (m & 1);
    return (m & 2) ? N / 2 + f : f;
}

// One workgroup per record: 256 words, then the pairs (s, z).  What lies behind K is zero.
__global__ __launch_bounds__(256) void w4_pack_kernel(const uint8_t *__restrict__ codes, const __half *__restrict__ scales,
                                                      const __half *__restrict__ zeros, uint8_t *__restrict__ dst, int N, int K,
                                                      int group, int gate_up, int record, int n_kb) {
    const int nt = blockIdx.x / n_kb, kb = blockIdx.x % n_kb, tid = threadIdx.x;
    uint8_t *rec = dst + (size_t)blockIdx.x * record;
    {
        const int c = tid >> 6, m = (tid >> 2) & 15, i = tid & 3, k = kb * 128 + 32 * i + 8 * c;
        unsigned out = 0;
        if (k < K) {
            const unsigned w = *(const unsigned *)(codes + ((size_t)w4_source_row(nt, m, N, gate_up) * K + k) / 2);
#pragma unroll
            for (int e = 0; e < 8; ++e) out |= ((w >> (4 * e)) & 15u) << (4 * ((e >> 1) + 4 * (e & 1)));
        }
        ((unsigned *)rec)[tid] = out;
    }
    const int ng = 128 / group;
    if (tid < ng * 16) {
        const int g = kb * ng + tid / 16, m = tid & 15;
        unsigned p = 0;
        if (g < K / group) {
            const size_t at = (size_t)w4_source_row(nt, m, N, gate_up) * (K / group) + g;
            p = (unsigned)__half_as_ushort(scales[at]) | (unsigned)__half_as_ushort(zeros ? zeros[at] : __float2half_rn(8.f)) << 16;
        }
        ((unsigned *)(rec + 1024))[tid] = p;
    }
}

__device__ float w4_dot(const W4Gemm &a, int m, int n_tile, int row) {
    const int n_kb = w4_kblocks(a.K), record = w4_record(a.group);
    float acc = 0.f;
    for (int k0 = 0; k0 < a.K; k0 += a.group) {
        const uint8_t *rec = a.W + ((size_t)n_tile * n_kb + (k0 >> 7)) * record;
        const unsigned p = ((const unsigned *)(rec + 1024))[((k0 & 127) / a.group) * 16 + row];
        const float s = __half2float(__ushort_as_half((unsigned short)(p & 0xffff))), z = __half2float(__ushort_as_half((unsigned short)(p >> 16)));
        float part = 0.f;
        for (int k = k0; k < k0 + a.group; k += 8) {
            const unsigned w = ((const unsigned *)rec)[(((k & 31) >> 3) * 16 + row) * 4 + ((k & 127) >> 5)];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                part += __bfloat162float(a.A[(size_t)m * a.K + k + e]) * ((float)((w >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15) - z);
        }
        acc += s * part;
    }
    return acc;
}

// A thread per output.
__global__ __launch_bounds__(256) void w4_gemm_kernel(W4Gemm a) {
    const int n_out = a.epi == EPI_SWIGLU ? a.N / 2 : a.N;
    const long at = (long)blockIdx.x * 256 + threadIdx.x;
    if (at >= (long)a.M * n_out) return;
    const int m = (int)(at / n_out), n = (int)(at % n_out);
    if (a.epi == EPI_SWIGLU) {
        const int f = n & 7, row = (f >> 1) * 4 + (f & 1);
        const float g = w4_dot(a, m, n >> 3, row), u = w4_dot(a, m, n >> 3, row + 2);
        ((bf16 *)a.out)[at] = __float2bfloat16(g / (1.f + expf(-g)) * u);
    } else {
        const float y = w4_dot(a, m, n >> 4, n & 15);
        ((float *)a.out)[at] = a.epi == EPI_RESID_F32 ? a.resid[at] + y : y;
    }
}

}  // namespace

hipError_t launch_w4_pack(const uint8_t *codes, const __half *scales, const __half *zeros, uint8_t *dst, int N, int K, int group,
                          int gate_up, hipStream_t s) {
    const int n_kb = w4_kblocks(K);
    w4_pack_kernel<<<(N / 16) * n_kb, 256, 0, s>>>(codes, scales, zeros, dst, N, K, group, gate_up, w4_record(group), n_kb);
    return hipGetLastError();
}

hipError_t launch_w4_gemm(const W4Gemm &a, hipStream_t s) {
    const long n = (long)a.M * (a.epi == EPI_SWIGLU ? a.N / 2 : a.N);
    w4_gemm_kernel<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cs
