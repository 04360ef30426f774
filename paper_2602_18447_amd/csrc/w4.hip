// Products of up to 128 rows with 4-bit weights.  Record format: confspec_int4.h, kernels.h.
#include "kernels.h"
#include <algorithm>

namespace cs {

namespace {

// Row of the matrix that is row m of the 16 of tile nt.  A gate/up matrix has eight gate rows and their eight up rows in a
// tile, so that a lane finds the other half of its pair eight lanes away.
__device__ __forceinline__ int w4_source_row(int nt, int m, int N, int gate_up) {
    if (!gate_up) return nt * 16 + m;
    const int f = nt * 8 + (m & 7);
    return (m & 8) ? N / 2 + f : f;
}

// One workgroup per record: 256 words, then the pairs (s, z / 16) of row 0's groups, row 1's, ...  What lies behind K is zero.  Done once
// per matrix: N = 55296, K = 5120 (142 MB of codes, 301 MB in all) 149 us.
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
        const int m = tid / ng, g = kb * ng + tid % ng;
        unsigned p = 0;
        if (g < K / group) {
            const size_t at = (size_t)w4_source_row(nt, m, N, gate_up) * (K / group) + g;
            const float z = zeros ? __half2float(zeros[at]) : 8.f;
            p = (unsigned)__half_as_ushort(scales[at]) | (unsigned)__half_as_ushort(__float2half_rn(z * 0.0625f)) << 16;
        }
        ((unsigned *)(rec + 1024))[tid] = p;
    }
}

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// Eight codes as bfloat16 16 + c: element 2 k and 2 k + 1 are nibbles k and k + 4.
struct CodeBits { unsigned mask, one; };   // in registers: one and-or takes both only if neither is a literal
__device__ __forceinline__ CodeBits code_bits() {
    CodeBits b;
    asm("s_mov_b32 %0, 0x780078" : "=s"(b.mask));
    asm("v_mov_b32 %0, 0x41804180" : "=v"(b.one));
    return b;
}
__device__ __forceinline__ bf16x8 code_operand(unsigned w, CodeBits b) {
    const unsigned M = b.mask, C = b.one;
    const u32x4 r = {((w << 3) & M) | C, ((w >> 1) & M) | C, ((w >> 5) & M) | C, ((w >> 9) & M) | C};
    return __builtin_bit_cast(bf16x8, r);
}

// A wavefront has 16 MT rows of A, 16 NT rows of W and every W-th block of 128 k; the wavefronts of a workgroup have the same
// rows and add up in LDS, in a fixed order.
//  * A record's codes are the second operand of four 16x16x32 products as they lie in memory, 16 bytes a lane, a code c as
//    the bfloat16 16 + c (its four bits put into the mantissa of 16), which is exact.  Before them goes a product with
//    -16 everywhere: it takes the offset out, and leaves -16 sum(a) of the group, which z / 16 is multiplied by.
//  * A lane has one row of W and four rows of A in the result, so that a group costs two multiply-adds a result, which take s and z
//    as the halves they are: sum += s (part - z sum(a)).
// Bound by the bytes of W while rows are few; every workgroup reads its rows of A from L2.  N = 55296, K = 5120, groups of 128, one row: 24.8
// us (6.1 TB/s, the weights come from the last-level cache; 30 with other weights each time, 5.0).  N = 5120, K = 27648, groups of 64, 8
// rows: 19.2 us (4.2 TB/s; 24.2), as its 160 tiles of 32 rows leave 96 CUs without.  72 rows, N = 7168, K = 5120, groups of 32: 22.4 us, in
// which no pipe is full (vector 43 %, matrix 15 %, wavefronts wait a third of their time): a block of k is load, stage, unpack and product in
// turn, with no load in flight meanwhile, every wavefront stages rows of A of its own, and each tile of W reads all of A again.
template <int NG>
struct Params;
template <> struct Params<1> { typedef unsigned T; static __device__ unsigned get(T p, int) { return p; } };
template <> struct Params<2> { typedef uint2 T; static __device__ unsigned get(T p, int g) { return g ? p.y : p.x; } };
template <> struct Params<4> { typedef u32x4 T; static __device__ unsigned get(T p, int g) { return p[g]; } };

// Row m of A times row n15 of the 16 whose records begin at `tile`, weights and sums as the definition has them, group by group.  A lane
// alone, for results that are no finite numbers otherwise: a row with an infinity in the last of K = 5120 makes a product take 0.3 ms instead
// of 0.03 (N = 55296), a row of NaN no longer.
__device__ __forceinline__ float w4_product(const bf16 *A, const uint8_t *tile, int m, int n15, int K, int ng) {
    const bf16 *a = A + (size_t)m * K;
    const int words = 4 / ng, n_groups = K / 32 / words;
    float sum = 0.f;
#pragma unroll 1
    for (int g = 0; g < n_groups && sum == sum; ++g) {        // (what is added to a NaN is NaN)
        const uint8_t *rec = tile + (size_t)(g / ng) * (1024 + 64 * ng);
        const f16x2 sz = __builtin_bit_cast(f16x2, *(const unsigned *)(rec + 1024 + (n15 * ng + g % ng) * 4));
        const float s = (float)sz[0], z = 16.f * (float)sz[1];
        float part = 0.f;
#pragma unroll 1
        for (int at = 0; at < 4 * words; ++at) {          // words of eight codes, k ascending: i = at / 4 of the group's, c = at % 4
            const int i = g % ng * words + at / 4, c = at % 4;
            const unsigned w = *(const unsigned *)(rec + ((c * 16 + n15) * 4 + i) * 4);
            const u32x4 v = *(const u32x4 *)(a + (size_t)g * 32 * words + 8 * at);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                part = fmaf(__uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16), s * ((float)((w >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15u) - z), part);
        }
        sum += part;
    }
    return sum;
}

constexpr int max_waves(int MT) { return MT == 1 ? 16 : 8; }   // of a workgroup: what the registers of a wavefront leave room for

// Loads of 16, 8 or 4 bytes from a wave-uniform base plus a byte offset per lane; offsets at or past the end read zeros, and
// touch no memory: so blocks behind the last one need no case of their own.
struct Loads {
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ Loads(const void *base, unsigned bytes) : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00020000)) {}
    __device__ void get(unsigned off, u32x4 &v) const { v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)off, 0, 0)); }
    __device__ void get(unsigned off, uint2 &v) const { v = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, (int)off, 0, 0)); }
    __device__ void get(unsigned off, unsigned &v) const { v = __builtin_amdgcn_raw_buffer_load_b32(rsrc, (int)off, 0, 0); }
};
constexpr unsigned PAST_END = 0x80000000u;

// AL: loads of four rows of A each a block takes, at least as many as there are rows.
template <int NT, int NG>
struct BlockW {                       // operands of one block of k as they come from memory
    u32x4 w[NT];
    typename Params<NG>::T p[NT];
};
template <int AL>
struct BlockA { u32x4 v[AL]; };

template <int MT, int AL, int NT, int NG>
__global__ __launch_bounds__(64 * max_waves(MT)) void w4_gemm_kernel(W4Gemm g, int n_mb, int W) {
    extern __shared__ u32x4 s_mem[];
    constexpr int REC = 1024 + 64 * NG;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n15 = lane & 15, kg = lane >> 4;
    const int mb = blockIdx.x % n_mb, nb = blockIdx.x / n_mb, m0 = mb * 16 * MT, t0 = nb * NT, n_tiles = g.N >> 4, n_kb = w4_kblocks(g.K);
    const unsigned w_at = lane * 16, p_at = 1024 + n15 * 4 * NG, tile_bytes = (unsigned)n_kb * REC;
    const Loads A(g.A, (unsigned)g.M * (unsigned)g.K * 2u), Wt(g.W + (size_t)t0 * tile_bytes, (unsigned)min(NT, n_tiles - t0) * tile_bytes);
    unsigned a_at[AL];                // byte offsets of the lane's rows of A (W4_MAX_K keeps the matrix below 2^31 bytes)
#pragma unroll
    for (int j = 0; j < AL; ++j) a_at[j] = (unsigned)min(m0 + 4 * j + kg, g.M - 1) * (unsigned)g.K * 2u;
    u32x4 *const s_a = s_mem + wave * MT * 256;
    f32x4 sum[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const CodeBits bits = code_bits();
    const u32x4 neg16_bits = {0xC180C180u, 0xC180C180u, 0xC180C180u, 0xC180C180u};
    const bf16x8 neg16 = __builtin_bit_cast(bf16x8, neg16_bits);

    auto load_a = [&](BlockA<AL> &b, int kb) {
        const unsigned k = (unsigned)kb * 256u + 16u * n15, at = (int)k < 2 * g.K ? k : PAST_END;      // (K a multiple of 32: 64 bytes)
#pragma unroll
        for (int j = 0; j < AL; ++j) A.get(a_at[j] + at, b.v[j]);
    };
    auto load_w = [&](BlockW<NT, NG> &b, int kb) {
        const unsigned rec = kb < n_kb ? (unsigned)kb * REC : PAST_END;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            Wt.get(rec + t * tile_bytes + w_at, b.w[t]);
            Wt.get(rec + t * tile_bytes + p_at, b.p[t]);
        }
        __builtin_amdgcn_sched_barrier(0);       // (loads stay ahead of the products before them in time)
    };
    // Rows of A: 16 lanes have 256 consecutive bytes of a row, the operand wants a row a lane; through LDS, where row r keeps
    // its 16-byte piece v at v ^ r % 16: 16 lanes then meet all banks both ways.
    auto stage = [&](const BlockA<AL> &b) {
#pragma unroll
        for (int j = 0; j < AL; ++j) s_a[(4 * j + kg) * 16 + (n15 ^ ((4 * j + kg) & 15))] = b.v[j];
        __builtin_amdgcn_wave_barrier();
    };
    auto compute = [&](const BlockW<NT, NG> &b) {
        bf16x8 a[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) a[m][i] = __builtin_bit_cast(bf16x8, s_a[(16 * m + n15) * 16 + ((4 * i + kg) ^ n15)]);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int q = 0; q < NG; ++q) {
            f32x4 off[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                off[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 4 / NG; ++i) off[m] = mma(a[m][q * (4 / NG) + i], neg16, off[m]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                f32x4 part[MT];
#pragma unroll
                for (int i = 0; i < 4 / NG; ++i) {
                    const bf16x8 c = code_operand(b.w[t][q * (4 / NG) + i], bits);
#pragma unroll
                    for (int m = 0; m < MT; ++m) part[m] = mma(a[m][q * (4 / NG) + i], c, i == 0 ? off[m] : part[m]);
                }
                const f16x2 sz = __builtin_bit_cast(f16x2, Params<NG>::get(b.p[t], q));
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[m][t][r] = fmaf((float)sz[0], fmaf((float)sz[1], off[m][r], part[m][r]), sum[m][t][r]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // One tile of rows: the next block is asked for as soon as A's registers are free, and the registers for W are there twice (with a
    // second set for A, asked for a block earlier: 8.9 us for 8.1, 16 rows, N = 17920, K = 1536, groups of 64).  More tiles have no registers
    // for that, nor time to win: 72 rows, N = 7168, K = 5120, groups of 32, tiles of 3 x 2: 23.4 us with, 23.9 without.
    BlockA<AL> x;
    BlockW<NT, NG> w0;
    if constexpr (MT == 1) {
        BlockW<NT, NG> w1;
        load_a(x, wave);
        load_w(w0, wave);
        for (int kb = wave; kb < n_kb; kb += 2 * W) {
            stage(x);
            load_a(x, kb + W);
            load_w(w1, kb + W);
            compute(w0);
            if (kb + W >= n_kb) break;
            stage(x);
            load_a(x, kb + 2 * W);
            load_w(w0, kb + 2 * W);
            compute(w1);
        }
    } else {
        for (int kb = wave; kb < n_kb; kb += W) {
            load_a(x, kb);
            load_w(w0, kb);
            stage(x);
            compute(w0);
        }
    }
    f32x4 *const s_part = (f32x4 *)s_mem;
    if (W > 1) __syncthreads();       // (A's places are written over)
    if (W > 1) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int t = 0; t < NT; ++t) s_part[((wave * MT + m) * NT + t) * 64 + lane] = sum[m][t];
        __syncthreads();
    }
    for (int tile = W > 1 ? wave : 0; tile < MT * NT; tile += W) {
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        if (W > 1) {
            for (int w = 0; w < W; ++w) y += s_part[(w * MT * NT + tile) * 64 + lane];
        } else {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    if (m * NT + t == tile) y = sum[m][t];
        }
        const int nt = t0 + tile % NT, m_first = m0 + 16 * (tile / NT) + 4 * kg;
        if (nt >= n_tiles) continue;
        // 16 + c and -16 cancel no infinity, and sums of 31 a leave fp32 before those of a weight times a do: where no finite number
        // came out, the definition says which other, or which one after all.
        unsigned again = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) again |= m_first + r < g.M && !(fabsf(y[r]) < INFINITY) ? 1u << r : 0u;
        for (; again; again &= again - 1) {
            const int first = __builtin_ctz(again);
            const float product = w4_product(g.A, g.W + (size_t)nt * tile_bytes, m_first + first, n15, g.K, NG);
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = r == first ? product : y[r];
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int m = m_first + r;
            if (g.epi == EPI_SWIGLU) {
                const float up = __shfl_xor(y[r], 8, 64);
                if (n15 < 8 && m < g.M)
                    ((bf16 *)g.out)[(size_t)m * (g.N >> 1) + nt * 8 + n15] = __float2bfloat16(y[r] / (1.f + __expf(-y[r])) * up);
            } else if (m < g.M) {
                const size_t at = (size_t)m * g.N + nt * 16 + n15;
                ((float *)g.out)[at] = g.epi == EPI_RESID_F32 ? g.resid[at] + y[r] : y[r];
            }
        }
    }
}

template <int MT, int AL, int NT, int NG>
hipError_t launch_group(const W4Gemm &a, int W, hipStream_t s) {
    const int n_mb = (a.M + 16 * MT - 1) / (16 * MT), n_nb = (a.N / 16 + NT - 1) / NT;
    const size_t lds = (size_t)W * MT * 1024 * std::max(4, NT);        // rows of A, then partial sums
    if (lds > 65536) {
        static std::atomic<uint32_t> set{0};
        if (hipError_t e = set_dynamic_lds_once(set, (const void *)w4_gemm_kernel<MT, AL, NT, NG>, max_waves(MT) * MT * 1024 * std::max(4, NT))) return e;
    }
    w4_gemm_kernel<MT, AL, NT, NG><<<dim3((unsigned)n_mb * (unsigned)n_nb), dim3(64 * W), lds, s>>>(a, n_mb, W);
    return hipGetLastError();
}
template <int MT, int AL, int NT>
hipError_t launch(const W4Gemm &a, int W, hipStream_t s) {
    return a.group == 128 ? launch_group<MT, AL, NT, 1>(a, W, s) : a.group == 64 ? launch_group<MT, AL, NT, 2>(a, W, s) : launch_group<MT, AL, NT, 4>(a, W, s);
}

}  // namespace

hipError_t launch_w4_pack(const uint8_t *codes, const __half *scales, const __half *zeros, uint8_t *dst, int N, int K, int group,
                          int gate_up, hipStream_t s) {
    const int n_kb = w4_kblocks(K);
    w4_pack_kernel<<<(N / 16) * n_kb, 256, 0, s>>>(codes, scales, zeros, dst, N, K, group, gate_up, w4_record(group), n_kb);
    return hipGetLastError();
}

// Which rows of A and of W a workgroup takes, and how many wavefronts share its k.  Up to 16 rows the bytes of W bound the product:
// 32 rows of W a workgroup once there are 256 tiles of 16 (N = 5120, K = 27648, 8 rows, groups of 64: 24.2 us, with 16 rows of W 29.9;
// N = 1536, K = 8960, one row: 7.2, with 16 rows 5.5), 4 wavefronts from 512 workgroups on (N = 55296, K = 5120, one row: 29.6, 8 32.8), 8 from
// 256, else 16 (160 workgroups, the first of these: 19.2, 8 21.8 on weights read just before; 24.2, 22.8 on others), if there are as many
// blocks of k (N = 5120, K = 1408, 4 rows: 8 wavefronts 4.2, 11 4.4).
// More rows on a small matrix are bound by what a workgroup can fetch, and tiles of 1 x 1 or 1 x 2 make the most workgroups, up to one a CU.
// Measured (us) for 1x1, 1x2 and 2x2 with 8 wavefronts, at so many tiles of 16 x 16: 34 (25 rows, N = 272, K = 17824, groups of 32): 12.7,
// 17.1, 28.3;  256 (20, 2048, 4096, 128): 5.5, 6.0, 8.0;  288 (40, 1536, 4096, 64): 7.8, 6.4, 8.2;  512 (20, 4096, 2048, 64): 6.0, 5.3, 6.0;
// 640 (30, 5120, 5120, 128): 16.7, 12.3, 10.9;  768 (128, 1536, 8960, 128): 21.5, 17.3, 14.9.
// Others take what a wavefront does in a block, one thing after the other: the tile with the least of w4_cost, in rounds of 256 workgroups.  Measured (us)
// for 2x2, 2x4, 3x2, 3x4, 4x4 tiles of 16 (4x4 with groups of 32 keeps one register in memory): 72 rows, N = 7168, K = 5120, groups of 128: 21.0, 19.9, 19.8, 16.2, 19.8;  48, 5120, 5120, 64:
// 15.6, 14.4, 13.8, 17.9, -;  128, 1536, 8960, 128: 14.7, 18.3, 17.3, -, -;  128, 55296, 5120, 128: 166, 131, -, 139, 120.
struct W4Tile { int mt, nt, W; };

int w4_cost(int mt, int nt, int ng) {    // issue cycles of a wavefront's block, in vector instructions: rows of A; unpacking; sums and products
    return mt * 46 + nt * 32 + mt * nt * (8 * ng + 8) + 40;
}

W4Tile w4_tile(int M, int N, int K, int group) {
    const int tiles = N / 16, n_kb = w4_kblocks(K);
    const long small = (long)((M + 15) / 16) * tiles;
    W4Tile t = {1, small <= 256 ? 1 : 2, 8};
    if (M <= 16) {
        t.nt = tiles >= 256 ? 2 : 1;
        const long groups = (tiles + t.nt - 1) / t.nt;
        t.W = groups >= 512 ? 4 : groups >= 256 || n_kb < 16 ? 8 : 16;
    } else if (small > 512) {
        long best = -1;
        for (const auto &c : {W4Tile{2, 2, 0}, W4Tile{2, 4, 0}, W4Tile{3, 2, 0}, W4Tile{3, 4, 0}, W4Tile{4, 4, 0}}) {
            const long units = (long)((M + 16 * c.mt - 1) / (16 * c.mt)) * ((tiles + c.nt - 1) / c.nt);
            const long cost = (units + 255) / 256 * w4_cost(c.mt, c.nt, 128 / group);
            if (best < 0 || cost < best) {
                best = cost;
                t = c;
                t.W = units <= 256 ? 8 : 4;
            }
        }
    }
    t.W = std::min(t.W, n_kb);
    return t;
}

hipError_t launch_w4_gemm(const W4Gemm &a, hipStream_t s) {
    const W4Tile t = w4_tile(a.M, a.N, a.K, a.group);
    if (t.mt == 1 && a.M <= 4) return t.nt == 1 ? launch<1, 1, 1>(a, t.W, s) : launch<1, 1, 2>(a, t.W, s);
    if (t.mt == 1 && a.M <= 8) return t.nt == 1 ? launch<1, 2, 1>(a, t.W, s) : launch<1, 2, 2>(a, t.W, s);
    if (t.mt == 1) return t.nt == 1 ? launch<1, 4, 1>(a, t.W, s) : launch<1, 4, 2>(a, t.W, s);
    if (t.mt == 2) return t.nt == 2 ? launch<2, 8, 2>(a, t.W, s) : launch<2, 8, 4>(a, t.W, s);
    if (t.mt == 3) return t.nt == 2 ? launch<3, 12, 2>(a, t.W, s) : launch<3, 12, 4>(a, t.W, s);
    return launch<4, 16, 4>(a, t.W, s);
}

}  // namespace cs
