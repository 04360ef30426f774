// The paged cache in 4 bits: append of rotated keys and values, its rows as values, attention over it.  Page format:
// confspec_int4.h.
#include "kernels.h"
#include <algorithm>

namespace cs {

namespace {

__device__ __forceinline__ float bf16_f32(bf16 v) { return __bfloat162float(v); }

// Trace of packed token t, the largest b with cu[b] <= t, by a whole wavefront: 64 candidates a round instead of two (a round is a
// trip to L2; a call on few tokens is made of such trips).
__device__ __forceinline__ int trace_of(const int32_t *cu, int B, int t, int lane) {
    int lo = 0, n = B;
    while (n > 1) {
        const int step = (n + 63) >> 6, at = lane * step;
        const int found = __popcll(__ballot(at < n && cu[min(lo + at, B - 1)] <= t));
        const int skip = max(found - 1, 0) * step;
        lo += skip;
        n = min(step, n - skip);
    }
    return __builtin_amdgcn_readfirstlane(lo);
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

// x as a half, a zero without its sign: 0 is added after the rounding, as all from -2^-25 on rounds to -0.  (The compiler may not see
// where x comes from: of a rounding from 64 bits to fp32 and this one it would make one.)
__device__ __forceinline__ __half half_unsigned_zero(float x) {
    asm("" : "+v"(x));
    return __builtin_bit_cast(__half, (_Float16)((_Float16)x + (_Float16)0.f));
}

// Half a wavefront per head, eight heads a workgroup at a time, n_split workgroups per token; lane i of a half has elements 2 i, 2 i + 1
// and the 64 further ones they are paired with: minimum, maximum and the words of codes need exchanges inside the half only.
// Rotated: (x, y) -> (x cos - y sin, y cos + x sin), angle (L_b + i) theta^(-j / 64).  Angles, rotation and what decides between
// two codes in 64 bits.
// Bound by the bytes of qkv and of q, k, v where tokens are many: 4096 tokens, 40 heads on 8: 34 us for 181 MB (5.3 TB/s); by latency
// (length, block number, row) where they are few: one token 3.7 us, of 12 heads on 2.  A wavefront's 64 lanes take the token's 64 angles for
// all (2362 tokens, 12 heads on 2: 9.8 us; each half its own, 10.9).
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4Append a, int n_split) {
    const Kv4Batch &b = a.b;
    const int t = blockIdx.x / n_split, split = blockIdx.x % n_split, lane = threadIdx.x & 63, i2 = lane & 31, heads = a.Hq + 2 * b.Hkv;
    int h = split * 8 + (threadIdx.x >> 5);
    const float *src = a.qkv + (size_t)t * a.stride + 2 * i2;
    float2 lo = *(const float2 *)(src + (size_t)min(h, heads - 1) * 128), hi = *(const float2 *)(src + (size_t)min(h, heads - 1) * 128 + 64);
    const int trace = trace_of(b.cu, b.B, t, lane);
    const int i = min(max(t - b.cu[trace], 0), b.T - 1), row = min(max(b.plens[trace], 0), b.max_L) + i, slot = row & 15;
    const bool store = (!a.n_append || i < a.n_append[trace]) && row >> 4 < b.max_blocks;
    uint8_t *const pages = page_of(b, trace, row, 0);
    // the token's 64 angles, once: theta^(-j / 64) from the six powers theta^(-2^k / 64)
    __shared__ double2 s_turn[64];
    if (threadIdx.x < 64) {
        double f = 1.0, sn, cs;
#pragma unroll
        for (int k = 0; k < 6; ++k) f *= (lane >> k) & 1 ? a.theta_pow[k] : 1.0;
        sincos64((double)row * f, sn, cs);
        s_turn[lane] = make_double2(cs, sn);
    }
    __syncthreads();
    const double c0 = s_turn[2 * i2].x, s0 = s_turn[2 * i2].y, c1 = s_turn[2 * i2 + 1].x, s1 = s_turn[2 * i2 + 1].y;
    for (; h < heads; h += 8 * n_split) {
        float2 lo_next = lo, hi_next = hi;
        if (h + 8 * n_split < heads) {
            lo_next = *(const float2 *)(src + (size_t)(h + 8 * n_split) * 128);
            hi_next = *(const float2 *)(src + (size_t)(h + 8 * n_split) * 128 + 64);
        }
        if (h < a.Hq + b.Hkv) {
            const double x0 = lo.x, x1 = lo.y, y0 = hi.x, y1 = hi.y;
            lo = make_float2((float)(x0 * c0 - y0 * s0), (float)(x1 * c1 - y1 * s1));
            hi = make_float2((float)(y0 * c0 + x0 * s0), (float)(y1 * c1 + x1 * s1));
        }
        const bf16 r[4] = {__float2bfloat16(lo.x), __float2bfloat16(lo.y), __float2bfloat16(hi.x), __float2bfloat16(hi.y)};
        const bool is_k = h >= a.Hq && h < a.Hq + b.Hkv;
        const int hk = is_k ? h - a.Hq : h - a.Hq - b.Hkv;
        bf16 *dst = (h < a.Hq ? a.q + ((size_t)t * a.Hq + h) * 128 : (is_k ? a.k : a.v) + ((size_t)t * b.Hkv + hk) * 128) + 2 * i2;
        *(unsigned *)dst = (unsigned)__bfloat16_as_ushort(r[0]) | (unsigned)__bfloat16_as_ushort(r[1]) << 16;
        *(unsigned *)(dst + 64) = (unsigned)__bfloat16_as_ushort(r[2]) | (unsigned)__bfloat16_as_ushort(r[3]) << 16;
        if (h >= a.Hq && store) {
            // min and max of the row, its pair (s, z), the codes
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = bf16_f32(r[e]);
            // A NaN anywhere in the row: s and z are NaN, which is what the definition's minimum is (v_med3 below would take it for -65504).
            const unsigned long long nan_lanes = __ballot(__builtin_isunordered(x[0], x[1]) || __builtin_isunordered(x[2], x[3]));
            const bool nan = (unsigned)(nan_lanes >> (lane & 32)) != 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_fmed3f(x[e], -65504.f, 65504.f);
            float mn = fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) { mn = fminf(mn, __shfl_xor(mn, o, 64)); mx = fmaxf(mx, __shfl_xor(mx, o, 64)); }
            const __half zh = half_unsigned_zero(mn);
            const float z = __half2float(zh);
            const __half sh = half_unsigned_zero((float)(((double)mx - (double)z) / 15.0));
            const float s = __half2float(sh);
            float n[4];
            bool close = false;                                     // a quotient that is a tie within its error, 16 times a few 2^-24
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float quotient = (x[e] - z) / s;
                n[e] = rintf(quotient);
                close |= fabsf(fabsf(quotient - n[e]) - 0.5f) < 0x1p-17f;
            }
            if (__any(close))                                       // what is left of the element decides, in 64 bits
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const double left = fma(-(double)n[e], (double)s, (double)x[e] - (double)z), half = 0.5 * (double)s;
                    const bool odd = ((int)n[e] & 1) != 0;
                    if (left > half || (odd && left == half)) n[e] += 1.f;
                    else if (left < -half || (odd && left == -half)) n[e] -= 1.f;
                }
            unsigned c[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] = s > 0.f && !nan ? (unsigned)fminf(fmaxf(n[e], 0.f), 15.f) : 0u;
            const int e = 2 * (lane & 3);                           // place of the first of the lane's two in their word of eight
            unsigned w0 = is_k ? c[0] << k_shift(e) | c[1] << k_shift(e + 1) : (c[0] | c[1] << 4) << (4 * e);
            unsigned w1 = is_k ? c[2] << k_shift(e) | c[3] << k_shift(e + 1) : (c[2] | c[3] << 4) << (4 * e);
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) { w0 |= (unsigned)__shfl_xor((int)w0, o, 64); w1 |= (unsigned)__shfl_xor((int)w1, o, 64); }
            uint8_t *page = pages + (size_t)hk * KV4_PAGE;
            if (e == 0) {
                *(unsigned *)(page + (is_k ? k_word(slot, 2 * i2) : v_word(slot, 2 * i2))) = w0;
                *(unsigned *)(page + (is_k ? k_word(slot, 2 * i2 + 64) : v_word(slot, 2 * i2 + 64))) = w1;
            }
            if (i2 == 0)
                *(unsigned *)(page + (is_k ? KV4_KP : KV4_VP) + slot * 4) =
                    nan ? 0x7E007E00u : (unsigned)__half_as_ushort(sh) | (unsigned)__half_as_ushort(zh) << 16;
        }
        lo = lo_next;
        hi = hi_next;
    }
}

__device__ __forceinline__ float param_s(unsigned p) { return __half2float(__ushort_as_half((unsigned short)(p & 0xffff))); }
__device__ __forceinline__ float param_z(unsigned p) { return __half2float(__ushort_as_half((unsigned short)(p >> 16))); }

// Eight heads of a token a workgroup at a time, n_split workgroups per token, four heads at once: a wavefront has a head's key and value
// row, a thread half a word of it, so that a wavefront's stores are 512 consecutive bytes twice.  Bound by what it writes: 4096 tokens, 8 heads: 10.9 us for 38 MB (3.5 TB/s).
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Batch b, int n_split, float *__restrict__ k, float *__restrict__ v) {
    const int t = blockIdx.x / n_split, lane = threadIdx.x & 63, first = blockIdx.x % n_split * 8 + (threadIdx.x >> 6);
    const int trace = trace_of(b.cu, b.B, t, lane);
    const int row = min(max(b.plens[trace], 0), b.max_L) + min(max(t - b.cu[trace], 0), b.T - 1), slot = row & 15;
    const int is_v = lane >> 5, d = (lane & 31) * 4;
    const uint8_t *pages = page_of(b, trace, row, 0);
    for (int h0 = first; h0 < b.Hkv; h0 += 8 * n_split)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int h = h0 + 4 * u;
            if (h >= b.Hkv) continue;
            const uint8_t *page = pages + (size_t)h * KV4_PAGE;
            const unsigned w = *(const unsigned *)(page + (is_v ? v_word(slot, d & ~7) : k_word(slot, d & ~7)));
            const unsigned p = *(const unsigned *)(page + (is_v ? KV4_VP : KV4_KP) + slot * 4);
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = fmaf(param_s(p), (float)((w >> (is_v ? 4 * ((d & 4) + e) : k_shift((d & 4) + e))) & 15), param_z(p));
            *(float4 *)((is_v ? v : k) + ((size_t)t * b.Hkv + h) * 128 + d) = make_float4(x[0], x[1], x[2], x[3]);
        }
}

// ---- attention ----
//
// A wavefront takes 16 NQ query rows of one (trace, kv head) - row = token * G + q head - and walks its share of the keys in
// chunks of 32 tokens: two pages of the cache, then 32 tokens of the suffix at a time.  It shares nothing with other
// wavefronts until the end and keeps its own (maximum, sum, O).
//  * Scores S^T = K Q^T: a page's key codes are the first operand of four 16x16x32 products as they lie in memory, 16
//    bytes a lane.  A code enters as a half below the normal range, its four bits alone: c 2^-24, or c 2^-20 where they stay in the
//    next four bits, and such elements of q are 1/16 of what they are: two of four codes need no shift.  q is a half too, times a
//    power of two of its row that brings its largest element to 2^13 .. 2^14: exact but for elements 2^-27 times smaller.  A lane then has
//    four keys of one query row: score = s sum + z sum(q), two multiply-adds that take s and z as the halves they are.
//  * O^T = V^T P^T: the lane's four keys of both pages are the eight consecutive k of the second operand as they are, and
//    a page's value codes lie in memory such that a lane's 16 bytes are those four tokens of eight columns.  Codes enter as
//    the keys' do, the probability as the half p s; z is added to the row's sum.  The lane has 32 columns of its one query row,
//    so scaling, sums and output need nothing of other lanes.
//    The rounding of p s moves what a row adds by less than p 15 2^-11 s, where the row's own step is p s.  Measured (48 traces of 2000 to 16384
//    tokens; 16 of steps of 32 to 256): outputs are 1.75e-3, 1.73e-3 (rms) from 64 bits, with probabilities in fp32 1.66e-3, most of it the
//    rounding to bf16.  A second half for what the first drops brings 1.66e-3, in 100 for 99 us and 157 for 135; codes counted from 8 (the sum
//    of the halves by one more product a row) 1.67e-3, in 99 and 138.5: not worth it beside steps of a fifteenth of a row's range.
//  * The running reference M of a row is a bound of score + exponent of s (p s is what must fit a half).  A chunk takes it as it is and
//    looks at the halves that come out; only where one has grown too large, M is raised, what was summed scaled and the chunk's
//    probabilities taken again.
//
// Bound by the cache's bytes when rows are few (136 bytes a token and head: 48 traces of 2000 to 16384 tokens, 40 heads on 8: 94 us for
// 478 MB, 5.1 TB/s, and 5.4 to join the pieces), by the vector pipe when they are many (16 traces of 32 to 256 tokens on 512 to 8192, 12
// heads on 2: 138 us, 0.54 PFLOP/s; a chunk is 224 vector instructions and 32 products of 32 rows by 32 keys), by latency when the batch
// is small (one token on 2048: 8.7 us, and 3.5 to join).
constexpr int ATT_TRACES = 256;       // traces of one launch
struct AttnPlan4 {
    int32_t b0, nb;                   // traces
    uint32_t per, per_inv;            // chunks of keys of a piece at most, 2^32 / per rounded up
    int32_t n_items, n_records, n_merge_rows;
    int32_t swizzle;
};

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ unsigned lo_halves(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }   // b.lo : a.lo
__device__ __forceinline__ unsigned hi_halves(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
// Four pairs of codes as halves: nibbles 0 and 2 of each 16 bits times 2^-24, nibbles 1 and 3 times 2^-20.
__device__ __forceinline__ u32x4 code_halves(unsigned w) {
    const unsigned u = w >> 8;
    return u32x4{w & 0x000F000Fu, w & 0x00F000F0u, u & 0x000F000Fu, u & 0x00F000F0u};
}
__device__ __forceinline__ unsigned pack_f16(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, f16x2));
}
__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ float max_over_g(float v) {       // over lanes l, l ^ 16, l ^ 32, l ^ 48
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_over_g(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

constexpr float SCALE_LOG2 = 0.08838834764831845f * 1.4426950408889634f;
// References: M bounds score + exponent field of s (15 where s is 1), all in powers of two, where it is raised; p = 2^(score - M + REF).
// Then p s is below 2^7, whatever the rows' s are; it may grow to W_ROOM = 2^15 (a half ends at 2^16), p (where s is 0) and its sum to
// L_ROOM, and the suffix's scores beyond M by M_ROOM, before M is raised again.
constexpr float M_NONE = -3e38f, M_ROOM = 8.f, REF = 20.f, E_ONE = 15.f, L_ROOM = 0x1p60f;
constexpr _Float16 W_ROOM = 32768;
// Where scores are beyond BIG, they are rounded before M is taken off (below, a multiply-add does both), M bounds score + E_BIG, whatever s
// is (p s < 2^14 still), and p is held at 2^(REF - E_BIG).  From 2^27 on, where E_BIG would be lost in M's own rounding, M bounds the score
// alone, and that hold is what bounds p, for all alike: equal scores keep equal weights.
constexpr float BIG = 16384.f, E_BIG = 22.f;
__device__ __forceinline__ float big_bound(float s) { return fabsf(s) < 0x1p27f ? s + E_BIG : s; }
// Sums of the cached tokens' value product are of so many units in even and in odd columns.
constexpr float EVEN_UNITS = 16777216.f, ODD_UNITS = 1048576.f;

// Loads of 16 bytes from a wave-uniform base plus a byte offset per lane; offsets at or past the end read zeros.
struct Loads {
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ Loads(const void *base, unsigned bytes) : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00020000)) {}
    __device__ u32x4 get(unsigned off) const { return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)off, 0, 0)); }
};

// What a wavefront needs of two pages; a lane's part of the pairs (s, z) are those of its four keys.
struct Chunk4 {
    u32x4 k[2], v[2], kp[2], vp[2];
};

template <int NQ>
struct Rows4 {                        // state of a wavefront's rows: a lane has row lane % 16 of each 16
    f16x8 q[NQ][4];                   // times a power of two of the row; elements 2, 3, 6, 7 of eight 1/16 of it
    float scale[NQ];                  // log2(e) / sqrt(128), that power and the codes' 2^-24 taken out
    float q_sum[NQ], m[NQ], l[NQ], zs[NQ];      // q_sum: sum(q) in the units of the product
    f32x4 o[NQ][8];                   // [j][r]: column 32 (lane / 16) + 8 r + j
};

// 2^x, x <= 0, never 0: what a sum is scaled by where the reference moves up.  A weight is positive however small, and takes an infinity
// along; numbers times 2^-126 are lost beside those that raised the reference.
__device__ __forceinline__ float scale_down(float x) { return fmaxf(__builtin_amdgcn_exp2f(x), 0x1p-126f); }

// Raises the references to the rows' largest score + exponent (t_max: the lane's).
template <int NQ>
__device__ __forceinline__ void raise(Rows4<NQ> &R, const float (&t_max)[NQ]) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const float m = fmaxf(R.m[i], max_over_g(t_max[i])), f = scale_down(R.m[i] - m);
        R.m[i] = m;
        R.l[i] *= f;
        R.zs[i] *= f;
#pragma unroll
        for (int j = 0; j < 8; ++j) R.o[i][j] *= f;
    }
}

__device__ __forceinline__ float mix(unsigned p, float a, float b) { return fmaf((float)__builtin_bit_cast(f16x2, p)[0], a, b); }    // s a + b
__device__ __forceinline__ float mix_z(unsigned p, float a, float b) { return fmaf((float)__builtin_bit_cast(f16x2, p)[1], a, b); }

// p = 2^score of the lane's eight keys of a row, p s as halves, sums of p and p z onto l0 and z0.
template <typename F>
__device__ __forceinline__ void probabilities(f16x8 &w, float &l, float &zs, float l0, float z0, const u32x4 (&vp)[2], F score) {
    l = l0;
    zs = z0;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float p = __builtin_amdgcn_exp2f(score(x, r));
            l += p;
            zs = mix_z(vp[x][r], p, zs);
            w[4 * x + r] = (_Float16)mix(vp[x][r], p, 0.f);
        }
}

// 32 cached tokens, of which the first n_valid count; what is stored for the others may be anything.
template <int NQ>
__device__ __forceinline__ void cached_chunk(Rows4<NQ> &R, const Chunk4 &c, int n_valid, int g, bool first, bool &big) {
    f32x4 sc[NQ][2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f16x8 a = __builtin_bit_cast(f16x8, code_halves(c.k[x][i]));
#pragma unroll
            for (int n = 0; n < NQ; ++n) sc[n][x] = mma(a, R.q[n][i], i == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sc[n][x]);
        }
    u32x4 vp[2] = {c.vp[0], c.vp[1]};
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int n = 0; n < NQ; ++n) sc[n][x][r] = mix(c.kp[x][r], sc[n][x][r], mix_z(c.kp[x][r], R.q_sum[n], 0.f));
    if (n_valid < 32)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * x + 4 * g + r >= n_valid) {
                    vp[x][r] = 0u;
#pragma unroll
                    for (int n = 0; n < NQ; ++n) sc[n][x][r] = -INFINITY;
                }
    // With the references as they are, unless that was too much for a half or an addend of the sums; most chunks end here.
    f16x8 w[NQ];
    float l[NQ], zs[NQ];
    bool over = big || first;         // (there is no reference before the first)
    if (!over) {
        f16x2 top = {0, 0};
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const float ref = REF - R.m[n];
            probabilities(w[n], l[n], zs[n], R.l[n], R.zs[n], vp, [&](int x, int r) { return fmaf(sc[n][x][r], R.scale[n], ref); });
#pragma unroll
            for (int e = 0; e < 8; e += 2) top = __builtin_elementwise_max(top, f16x2{w[n][e], w[n][e + 1]});
            over |= l[n] > L_ROOM;
        }
        over |= top[0] > W_ROOM || top[1] > W_ROOM;
    }
    if (__any(over)) {
#pragma clang fp contract(off)
        float t_max[NQ], s_max[NQ];
        bool beyond = false;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            t_max[n] = s_max[n] = -INFINITY;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    sc[n][x][r] *= R.scale[n];
                    s_max[n] = fmaxf(s_max[n], sc[n][x][r]);
                    t_max[n] = fmaxf(t_max[n], sc[n][x][r] + (float)((vp[x][r] >> 10) & 31u));
                }
            beyond |= fabsf(t_max[n]) > BIG && t_max[n] > M_NONE;
        }
        big |= (bool)__any(beyond);
        if (big)
#pragma unroll
            for (int n = 0; n < NQ; ++n) t_max[n] = big_bound(s_max[n]);
        raise<NQ>(R, t_max);
        const float most = big ? REF - E_BIG : INFINITY;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
            probabilities(w[n], l[n], zs[n], R.l[n], R.zs[n], vp, [&](int x, int r) { return fminf((sc[n][x][r] - R.m[n]) + REF, most); });
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        R.l[n] = l[n];
        R.zs[n] = zs[n];
    }
    unsigned lo[4], hi[4];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            lo[2 * x + r] = lo_halves(c.v[x][2 * r], c.v[x][2 * r + 1]);
            hi[2 * x + r] = hi_halves(c.v[x][2 * r], c.v[x][2 * r + 1]);
        }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        u32x4 col[4];                 // columns 4 h .. 4 h + 3
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const u32x4 v = code_halves(h ? hi[r] : lo[r]);
#pragma unroll
            for (int j = 0; j < 4; ++j) col[j][r] = v[j];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < NQ; ++n) R.o[n][4 * h + j] = mma(__builtin_bit_cast(f16x8, col[j]), w[n], R.o[n][4 * h + j]);
    }
}

// Eight values: a full exponent carries into its sign's place.
__device__ __forceinline__ unsigned exponent_full(u32x4 w) {
    unsigned any = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) any |= (w[e] & 0x7fff7fffu) + 0x00800080u;
    return any;
}

// Adds the values of tokens j_begin .. j_end - 1 that are not finite numbers to the rows that see them.  A probability is positive,
// so that an infinity or NaN is what its column becomes, whatever the probability.
template <int NQ>
__device__ __forceinline__ void add_not_finite(Rows4<NQ> &R, const bf16 *v, unsigned stride, int j_begin, int j_end, const int (&tok)[NQ], int g) {
#pragma unroll 1
    for (int j = j_begin; j < j_end; ++j) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const u32x4 w = *(const u32x4 *)(v + (uint64_t)(unsigned)j * stride + 32 * g + 8 * r);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const unsigned bits = e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16;
#pragma unroll
                for (int n = 0; n < NQ; ++n)
                    if ((bits & 0x7f800000u) == 0x7f800000u && j <= tok[n]) R.o[n][e][r] += __uint_as_float(bits);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Columns that came out as NaN, from the values of the tokens that were attended to: the two terms of a probability may have both
// signs or be 0, so that an infinity ends as NaN where the definition has an infinity.  (A NaN of the scores or of the cache is in R.l or
// R.zs too, and stays.)  One infinity among the first of 4096 tokens, 40 heads on 8: 0.76 ms, 0.45 without; a trace of NaN does not come here.
template <int NQ>
__device__ __forceinline__ void settle_not_finite(Rows4<NQ> &R, const bf16 *v, unsigned stride, int j0, int j_step, int j_end, int S, const int (&tok)[NQ], int n15, int g) {
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
            for (int r = 0; r < 4; ++r) R.o[n][j][r] = R.o[n][j][r] == R.o[n][j][r] ? R.o[n][j][r] : 0.f;
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll 1
    for (; j0 < j_end; j0 += j_step) {
        unsigned any = 0;
#pragma unroll
        for (int t = 0; t < 8; ++t) any |= exponent_full(*(const u32x4 *)(v + (uint64_t)(unsigned)min(j0 + 16 * (t >> 2) + 4 * g + (t & 3), S - 1) * stride + 8 * n15));
        if (__any((any & 0x80008000u) != 0u)) add_not_finite<NQ>(R, v, stride, j0, min(j0 + 32, S), tok, g);
    }
}

// Suffix tokens, 32 from j0 on, then from j0 + j_step, below j_end; k, v point at the trace's first token and the head, rows are `stride`
// elements apart; a row sees tokens up to its own (tok).  Products in bfloat16, probabilities in two terms; R.o is in units of 1.
// Values are asked for before the scores are taken, the next keys as soon as the registers of these are free.
template <int NQ>
__device__ __forceinline__ void attend_suffix(Rows4<NQ> &R, bool &big, const bf16 *q, const int (&q_row)[NQ], const bf16 *k, const bf16 *v, unsigned stride,
                                              int j0, int j_step, int j_end, int S, const int (&tok)[NQ], int n15, int g) {
    bf16x8 qb[NQ][4], kb[2][4];
    const int j_first = j0;
    bool whole = false;               // a chunk's values went into the products as they are
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) qb[n][i] = *(const bf16x8 *)(q + (size_t)q_row[n] * 128 + 8 * g + 32 * i);
    auto load_k = [&](int j) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) kb[x][i] = *(const bf16x8 *)(k + (uint64_t)(unsigned)min(j + 16 * x + n15, S - 1) * stride + 8 * g + 32 * i);
        __builtin_amdgcn_sched_barrier(0);
    };
    load_k(j0);
#pragma unroll 1
    for (; j0 < j_end; j0 += j_step) {
        u32x4 vw[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) vw[t] = *(const u32x4 *)(v + (uint64_t)(unsigned)min(j0 + 16 * (t >> 2) + 4 * g + (t & 3), S - 1) * stride + 8 * n15);
        __builtin_amdgcn_sched_barrier(0);
        f32x4 sc[NQ][2];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int n = 0; n < NQ; ++n) sc[n][x] = mma(kb[x][i], qb[n][i], i == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sc[n][x]);
        __builtin_amdgcn_sched_barrier(0);
        if (j0 + j_step < j_end) load_k(j0 + j_step);
        // A value that is not a finite number may only reach the rows that see its token, but a product takes 0 times it into every
        // row: where rows see a part of the tokens, such values are taken out, and added in the end.
        bool masked = false, bad = false;
#pragma unroll
        for (int n = 0; n < NQ; ++n) masked |= j0 + 31 > tok[n];
        if (!__any(masked)) {
            whole = true;
        } else {
            unsigned any = 0;
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int j = j0 + 16 * (t >> 2) + 4 * g + (t & 3);
#pragma unroll
                for (int n = 0; n < NQ; ++n)
                    if (j > tok[n]) sc[n][t >> 2][t & 3] = -INFINITY;
                if (j >= S) vw[t] = u32x4{0u, 0u, 0u, 0u};
                any |= exponent_full(vw[t]);
            }
            bad = __any((any & 0x80008000u) != 0u);
            if (bad)
#pragma unroll
                for (int t = 0; t < 8; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((vw[t][e] & 0x7f80u) == 0x7f80u) vw[t][e] &= 0xffff0000u;
                        if ((vw[t][e] & 0x7f800000u) == 0x7f800000u) vw[t][e] &= 0xffffu;
                    }
        }
        float t_max[NQ];
        bool beyond = false;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            t_max[n] = -INFINITY;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) t_max[n] = fmaxf(t_max[n], sc[n][x][r]);
            t_max[n] *= SCALE_LOG2;
            beyond |= fabsf(t_max[n]) > BIG && t_max[n] > M_NONE;
        }
        big |= (bool)__any(beyond);
        bool over = big;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            t_max[n] = big ? big_bound(t_max[n]) : t_max[n] + E_ONE;
            over |= t_max[n] > R.m[n] + M_ROOM;
        }
        if (__any(over)) raise<NQ>(R, t_max);
        if (big) {
#pragma clang fp contract(off)
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[n][x][r] = fminf((sc[n][x][r] * SCALE_LOG2 - R.m[n]) + REF, REF - E_BIG);
        } else {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const float ref = REF - R.m[n];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[n][x][r] = fmaf(sc[n][x][r], SCALE_LOG2, ref);
            }
        }
        u32x4 hi[NQ], lo[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    const float p0 = __builtin_amdgcn_exp2f(sc[n][x][r]), p1 = __builtin_amdgcn_exp2f(sc[n][x][r + 1]);
                    R.l[n] += p0;
                    R.l[n] += p1;
                    const unsigned h = pack_bf16(p0, p1);
                    hi[n][2 * x + (r >> 1)] = h;
                    lo[n][2 * x + (r >> 1)] = pack_bf16(p0 - __uint_as_float(h << 16), p1 - __uint_as_float(h & 0xffff0000u));
                }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u32x4 a;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                a[r] = j & 1 ? hi_halves(vw[2 * r][j >> 1], vw[2 * r + 1][j >> 1]) : lo_halves(vw[2 * r][j >> 1], vw[2 * r + 1][j >> 1]);
            const bf16x8 av = __builtin_bit_cast(bf16x8, a);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                R.o[n][j] = mma(av, __builtin_bit_cast(bf16x8, hi[n]), R.o[n][j]);
                R.o[n][j] = mma(av, __builtin_bit_cast(bf16x8, lo[n]), R.o[n][j]);
            }
        }
        if (bad) add_not_finite<NQ>(R, v, stride, j0, min(j0 + 32, S), tok, g);
    }
    if (whole) {
        bool lost = false;            // (where scores are NaN, so is the sum of the probabilities, and nothing can be settled)
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float all = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) all += R.o[n][j][r];
            lost |= all != all && R.l[n] == R.l[n];
        }
        if (__any(lost)) settle_not_finite<NQ>(R, v, stride, j_first, j_step, j_end, S, tok, n15, g);
    }
}

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ int dpp_add(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROW_MASK, 0xf, false); }
__device__ __forceinline__ int scan64(int v) {               // inclusive sums over the lanes
    v = dpp_add<0x111, 0xf>(v);                              // row_shr:1, 2, 4, 8 inside each 16 lanes
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);                              // row_bcast:15, row_bcast:31
    return dpp_add<0x143, 0xc>(v);
}

// Where an item of the launch (MERGE: a row of a trace that was cut) lies.  The list is never written out: every wavefront adds the
// traces' counts up, 64 at a time, from the lengths it needs anyway, so that a launch takes 256 traces and no list is copied for it.
// What the host counted (same arithmetic: count_items) bounds what is found.
struct Place4 {
    int trace, t0, S, L, P, n_tiles, local, first_record;
    bool found;
};
struct Count4 { int tiles, pieces, items, records, merge_rows; };
__host__ __device__ inline Count4 count_items(int L, int S, int G, int Hkv, int rows_log2, uint32_t per, uint32_t per_inv) {
    Count4 c;
    c.tiles = (int)(((long)G * S + (1 << rows_log2) - 1) >> rows_log2);
    // rounded up (one more than that, in places, where chunks go into the millions: nothing but this function decides it)
    c.pieces = (int)(((uint64_t)(((L + 31) >> 5) + ((S + 31) >> 5) + per - 1) * per_inv) >> 32);
    c.items = Hkv * c.tiles * c.pieces;
    c.records = c.pieces > 1 ? c.items : 0;
    c.merge_rows = c.pieces > 1 ? Hkv * G * S : 0;
    return c;
}
template <bool MERGE>
__device__ __forceinline__ Place4 find_item(const Kv4Batch &kv, const AttnPlan4 &plan, int G, int rows_log2, unsigned item, int lane) {
    int items0 = 0, records0 = 0;
    Place4 f = {};
    for (int k = 0; k < plan.nb; k += 64) {
        const int b = min(plan.b0 + min(k + lane, plan.nb - 1), kv.B - 1);
        const int c0 = kv.cu[b], c1 = kv.cu[b + 1], len = kv.plens[b];
        const int t0 = min(max(c0, 0), kv.T - 1), S = min(max(c1 - t0, 1), kv.T - t0), L = min(max(len, 0), kv.max_L);
        const Count4 c = count_items(L, S, G, kv.Hkv, rows_log2, plan.per, plan.per_inv);
        const bool in = k + lane < plan.nb;
        const int n = in ? (MERGE ? c.merge_rows : c.items) : 0, rec = in ? c.records : 0;
        const int n_sum = scan64(n), rec_sum = scan64(rec);
        const unsigned long long behind = __ballot((unsigned)(items0 + n_sum) > item);
        if (behind) {
            const int l = __builtin_ctzll(behind);
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
            f = Place4{min(plan.b0 + k + l, kv.B - 1), of(t0), of(S), of(L), of(c.pieces), of(c.tiles), (int)item - items0 - of(n_sum - n), records0 + of(rec_sum - rec), true};
            break;
        }
        items0 += __builtin_amdgcn_readlane(n_sum, 63);
        records0 += __builtin_amdgcn_readlane(rec_sum, 63);
    }
    return f;
}

constexpr int O_PAD = 132;            // floats from row to row of O in LDS

// WR x WK wavefronts: WR have different rows, WK of the same rows take different chunks of keys.
template <int NQ, int WR, int WK>
__global__ __launch_bounds__(WR * WK * 64, NQ == 1 && WK == 4 ? 3 : 2) void kv4_attn_kernel(Kv4Attn a, AttnPlan4 plan, float *part_o, float2 *part_ml) {
    constexpr int ROWS = 16 * NQ * WR, ROWS_LOG2 = __builtin_ctz(ROWS);
    __shared__ float s_o[WK > 1 ? WK * ROWS * O_PAD : 1];
    __shared__ float2 s_ml[WK > 1 ? WK * ROWS : 1];
    const Kv4Batch &kv = a.b;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WK, wk = wave % WK;
    const int n15 = lane & 15, g = lane >> 4;
    unsigned item = blockIdx.x;
    if (plan.swizzle) {               // workgroups are dealt out over 8 L2 caches: neighbours in the list, which share keys, to one
        const unsigned per = gridDim.x / 8, x = item % 8, rest = gridDim.x % 8;
        item = x * per + min(x, rest) + item / 8;
    }
    const int G = a.Hq / kv.Hkv;
    const Place4 f = find_item<false>(kv, plan, G, ROWS_LOG2, item, lane);
    if (!f.found) return;             // (only where device and host lengths differ; so are the record's bounds below)
    const int trace = f.trace, t0 = f.t0, S = f.S, L = f.L, n_rows = G * S, n_tiles = f.n_tiles, P = f.P;
    const int rt = f.local % n_tiles, piece = f.local / n_tiles % P, h = f.local / n_tiles / P;
    const int row0 = rt * ROWS + wr * 16 * NQ;

    Rows4<NQ> R;
    int tok[NQ], q_row[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int row = min(row0 + 16 * n + n15, n_rows - 1);
        tok[n] = row / G;
        q_row[n] = (t0 + tok[n]) * a.Hq + h * G + row % G;
        const bf16 *q = a.q + (size_t)q_row[n] * 128 + 8 * g;
        bf16x8 v[4];
        float sum = 0.f, top = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = *(const bf16x8 *)(q + 32 * i);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum += (float)v[i][e];
                top = fmaxf(top, fabsf((float)v[i][e]));
            }
        }
        // 2^(14 - x), where x is the exponent behind the row's largest element: between 2^114 and 2^-102
        const int x = min(max((int)(__float_as_uint(max_over_g(top)) >> 23) - 126, -100), 116);
        const float up = __uint_as_float((unsigned)(14 - x + 127) << 23);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) R.q[n][i][e] = (_Float16)((float)v[i][e] * (e & 2 ? up * 0.0625f : up));
        const float unit = __uint_as_float((unsigned)(x + 10 + 127) << 23);      // 2^24 / 2^(14 - x)
        R.scale[n] = SCALE_LOG2 * unit;
        R.q_sum[n] = sum_over_g(sum) * __uint_as_float((unsigned)(127 - x - 10) << 23);
        R.m[n] = M_NONE;
        R.l[n] = R.zs[n] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) R.o[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // chunks of this piece: cached ones first, then the suffix as far as the tile's last row sees it
    const int n_cached = (L + 31) >> 5, tok_hi = (min((rt + 1) * ROWS, n_rows) - 1) / G, n_all = n_cached + (tok_hi >> 5) + 1;
    const int c_begin = (int)((int64_t)n_all * piece / P), c_end = (int)((int64_t)n_all * (piece + 1) / P);
    const int c_stop = min(c_end, n_cached);
    bool big = false;                 // scores beyond BIG were met
    if (c_begin + wk < c_stop) {
        const int32_t *table = kv.table + (size_t)trace * kv.max_blocks;
        const uint8_t *head = kv.pages + (size_t)h * KV4_PAGE;
        const size_t block_bytes = (size_t)kv.Hkv * KV4_PAGE;
        const unsigned at16 = lane * 16, at_kp = KV4_KP + g * 16;
        // Block numbers of 32 chunks, two lanes each, and of the 32 after them; chunk i of this wavefront is c_begin + wk + i WK.
        auto block_ids = [&](int i0) {
            const int page = 2 * (c_begin + wk + WK * (i0 + (lane >> 1))) + (lane & 1);
            return table[min(page, kv.max_blocks - 1)];
        };
        int ids = block_ids(0), ids_next = block_ids(32);
        auto load = [&](Chunk4 &d, int i) {      // called with 0, 1, 2, ... (a chunk behind the last one reads zeros, and touches no memory)
            if (i && (i & 31) == 0) {
                ids = ids_next;
                ids_next = block_ids(i + 32);
            }
            const unsigned bytes = c_begin + wk + WK * i < c_stop ? KV4_PAGE : 0;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int id = min(max(__builtin_amdgcn_readlane(ids, 2 * (i & 31) + x), 0), kv.n_blocks - 1);
                const Loads page(head + (size_t)id * block_bytes, bytes);
                d.k[x] = page.get(at16);
                d.v[x] = page.get(KV4_V + at16);
                d.kp[x] = page.get(at_kp);
                d.vp[x] = page.get(KV4_VP - KV4_KP + at_kp);
            }
            __builtin_amdgcn_sched_barrier(0);   // (loads stay ahead of the products before them in time)
        };
        auto compute = [&](const Chunk4 &d, int i) {
            cached_chunk<NQ>(R, d, L - 32 * (c_begin + wk + WK * i), g, i == 0, big);
            __builtin_amdgcn_sched_barrier(0);
        };
        const int n = (c_stop - c_begin - wk + WK - 1) / WK;
        Chunk4 c0, c1;
        load(c0, 0);
        for (int i = 0; i < n; i += 2) {
            load(c1, i + 1);
            compute(c0, i);
            load(c0, i + 2);
            if (i + 1 < n) compute(c1, i + 1);
        }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int j = 0; j < 8; ++j) R.o[n][j] *= j & 1 ? ODD_UNITS : EVEN_UNITS;
    int c = c_begin + wk;
    if (c < c_stop) c += (c_stop - c + WK - 1) / WK * WK;
    const int c_last = min(c_end, n_cached + (min(row0 + 16 * NQ, n_rows) - 1) / G / 32 + 1);      // (as far as this wavefront's rows see)
    if (c < c_last)
        attend_suffix<NQ>(R, big, a.q, q_row, a.k + ((size_t)t0 * kv.Hkv + h) * 128, a.v + ((size_t)t0 * kv.Hkv + h) * 128, kv.Hkv * 128, 32 * (c - n_cached), 32 * WK,
                          32 * (c_last - n_cached), S, tok, n15, g);

    const bool direct = P == 1;
    const size_t rec = (size_t)f.first_record + ((size_t)(h * n_tiles + rt) * P + piece);
    if (!direct && rec >= (size_t)plan.n_records) return;
    auto store8 = [&](int tile_row, int col, const float (&o)[8], float m, float l, bool first) {
        const int row = rt * ROWS + tile_row;
        if (row >= n_rows) return;
        if (direct) {
            const float f = 1.f / l;
            const u32x4 r = {pack_bf16(o[0] * f, o[1] * f), pack_bf16(o[2] * f, o[3] * f), pack_bf16(o[4] * f, o[5] * f), pack_bf16(o[6] * f, o[7] * f)};
            *(u32x4 *)(a.out + ((size_t)(t0 + row / G) * a.Hq + h * G + row % G) * 128 + col) = r;
        } else {
            float *dst = part_o + (rec * ROWS + tile_row) * 128 + col;
            *(f32x4 *)dst = f32x4{o[0], o[1], o[2], o[3]};
            *(f32x4 *)(dst + 4) = f32x4{o[4], o[5], o[6], o[7]};
            if (first) part_ml[rec * ROWS + tile_row] = make_float2(m, l);
        }
    };
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const float l = sum_over_g(R.l[n]), zs = sum_over_g(R.zs[n]);
        const int row = wr * 16 * NQ + 16 * n + n15;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = R.o[n][j][r] + zs;
            if constexpr (WK == 1) {
                store8(row, 32 * g + 8 * r, o, R.m[n], l, g == 0 && r == 0);
            } else {
                float *dst = s_o + (wk * ROWS + row) * O_PAD + 32 * g + 8 * r;
                *(f32x4 *)dst = f32x4{o[0], o[1], o[2], o[3]};
                *(f32x4 *)(dst + 4) = f32x4{o[4], o[5], o[6], o[7]};
                if (g == 0 && r == 0) s_ml[wk * ROWS + row] = make_float2(R.m[n], l);
            }
        }
    }
    if constexpr (WK > 1) {
        __syncthreads();
        for (int at = tid; at < ROWS * 16; at += WR * WK * 64) {
            const int tile_row = at >> 4, col = (at & 15) * 8;
            float m = M_NONE;
#pragma unroll
            for (int w = 0; w < WK; ++w) m = fmaxf(m, s_ml[w * ROWS + tile_row].x);
            float l = 0.f, o[8] = {};
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float2 ml = s_ml[w * ROWS + tile_row];
                const float f = scale_down(ml.x - m);
                l += f * ml.y;
                const float *src = s_o + (w * ROWS + tile_row) * O_PAD + col;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] += f * src[e];
            }
            store8(tile_row, col, o, m, l, col == 0);
        }
    }
}

// One wavefront per (head, row) of the traces that were cut: a lane has two columns.  The sum over pieces of exp2(M_p - M) (O_p, l_p), M the
// largest of them; bound by its reads of O: 19884 rows of 128 in some 3 pieces 12 us, 1920 in some 5 pieces 5.4 us.
__global__ __launch_bounds__(256) void kv4_merge_kernel(Kv4Attn a, AttnPlan4 plan, int rows_log2, const float *__restrict__ part_o,
                                                        const float2 *__restrict__ part_ml) {
    const Kv4Batch &kv = a.b;
    const int lane = threadIdx.x & 63;
    const unsigned at = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (at >= (unsigned)plan.n_merge_rows) return;
    const int G = a.Hq / kv.Hkv;
    const Place4 f = find_item<true>(kv, plan, G, rows_log2, at, lane);
    if (!f.found) return;
    const int t0 = f.t0, n_rows = G * f.S, P = f.P, h = f.local / n_rows, row = f.local % n_rows, tile_rows = 1 << rows_log2;
    const size_t rec = (size_t)f.first_record + (size_t)(h * f.n_tiles + (row >> rows_log2)) * P;
    if (rec + P > (size_t)plan.n_records) return;
    const size_t first = rec * tile_rows + (row & (tile_rows - 1));
    const float *o = part_o + first * 128 + 2 * lane;
    const size_t step = (size_t)tile_rows * 128;
    // 64 pieces a round: a lane has the maximum and sum of one, and all their rows of O are asked for before they are needed
    float m = M_NONE, l = 0.f, o0 = 0.f, o1 = 0.f;
    for (int p0 = 0; p0 < P; p0 += 64) {
        const int n = min(64, P - p0);
        const float2 ml = lane < n ? part_ml[first + (size_t)(p0 + lane) * tile_rows] : make_float2(M_NONE, 0.f);
        float top = ml.x;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
        top = fmaxf(top, m);
        const float keep = scale_down(m - top), f = scale_down(ml.x - top);
        float sum = f * ml.y;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
        m = top;
        l = l * keep + sum;
        o0 *= keep;
        o1 *= keep;
        for (int p = 0; p < n; p += 4) {
            float2 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = p + u < n ? *(const float2 *)(o + (size_t)(p0 + p + u) * step) : make_float2(0.f, 0.f);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), min(p + u, n - 1)));
                if (p + u < n) {
                    o0 += w * v[u].x;
                    o1 += w * v[u].y;
                }
            }
        }
    }
    *(unsigned *)(a.out + ((size_t)(t0 + row / G) * a.Hq + h * G + row % G) * 128 + 2 * lane) = pack_bf16(o0 / l, o1 / l);
}

// The launches of a batch: up to ATT_TRACES traces each.
struct Launch4 {
    AttnPlan4 plan;
    int nq, wr, wk;
    int rows_log2() const { return __builtin_ctz(16 * nq * wr); }
    size_t record_rows() const { return (size_t)plan.n_records << rows_log2(); }
};
// Pieces are of 32 chunks at least: smaller ones bring the join, and its launch, to contexts that one piece finishes sooner.  Measured, us, with at
// least 16, 32 and 64 chunks: one token of 12 heads on 2, on 512 keys 9.8, 7.0, 7.0; 1024: 9.8, 10.3, 8.6; 2048: 10.9, 11.2, 11.9; 4096: 11.2,
// 11.9, 13.1; 8192: 12.4, 13.0, 14.2;  16 traces of one, 40 heads on 8, on 512: 10.6, 7.4, 7.4; 1024: 11.6, 11.4, 9.3; 8192: 30.3, 29.8, 30.7;
// 32 traces of 20 to 100 tokens on 100 to 900: 37.6, 27.3, 27.2.
// With eight wavefronts one workgroup fits a CU, and what does not fit at once waits for a whole item: as
// few items as there are CUs (one token on 16384 keys, 12 heads on 2: 13.7 us; in pieces of a power of two of chunks, which leave some CUs
// without, 18).  With four, two or three fit, and more items even out (16 traces of 32 to 256 tokens: 135 us, with 1024 items 141).
constexpr int ATT_MIN_CHUNKS = 32;
constexpr int att_slots(int wk) { return wk == 8 ? 256 : 1536; }

// Rows of a wavefront and wavefronts that share the keys.  32 rows halve the unpacking for each, 16 make more wavefronts; eight
// wavefronts finish an item sooner, four leave a batch with many items less to merge.  Measured, us (16 rows x 4, 16 x 8, 32 x 4, 32 x 8):
// 96 tokens on one context of 4096, 12 heads on 2: 16.8, 16.0, -, -;  32 traces of 1 to 7 tokens: 22.2, 21.4, -, -;  16 traces of 32 to 256
// tokens: 147, 210, 139, 169;  48 traces of one token, 40 heads on 8: 100, 111, -, -.
// Where no row has more than 16 chunks of keys and rows are many, sharing them costs more than it brings: four wavefronts of 32 rows each (32 x 4 and these):
// 64 traces of 100 to 256 tokens on 10 to 100, 12 heads on 2: 87, 55;  16 of 128 on 16: 20.8, 14.6;  32 of 20 to 100 on 100 to 900 (17
// chunks): 28.9, 32.9;  16 of 8 to 24 on 50 to 300, 40 heads on 8 (384 tiles): 12.4, 16.0.
void plan_launch(Launch4 &p, const int32_t *h_cu, const int32_t *h_lens, int b0, int nb, int Hq, int Hkv) {
    const int G = Hq / Hkv;
    int max_S = 0;
    int64_t units = 0, most = 0;      // tiles of 32 rows, chunks of the longest
    for (int b = b0; b < b0 + nb; ++b) {
        const int S = h_cu[b + 1] - h_cu[b];
        max_S = std::max(max_S, S);
        units += (int64_t)Hkv * (((int64_t)G * S + 31) / 32);
        most = std::max(most, ((int64_t)h_lens[b] + 31) / 32 + (S + 31) / 32);
    }
    p.nq = (int64_t)G * max_S <= 16 || units < 128 ? 1 : 2;
    p.wk = units >= 256 ? 4 : 8;
    p.wr = 1;
    if (p.nq == 2 && units >= 512 && most <= 16) p.wr = 4, p.wk = 1;
    const int slots = att_slots(p.wk);
    AttnPlan4 &a = p.plan;
    int64_t total = 0;                // chunks of all tiles
    for (int b = b0; b < b0 + nb; ++b) {
        const int S = h_cu[b + 1] - h_cu[b];
        total += (int64_t)Hkv * (((int64_t)G * S + (1 << p.rows_log2()) - 1) >> p.rows_log2()) * (((int64_t)h_lens[b] + 31) / 32 + (S + 31) / 32);
    }
    for (int64_t per = std::max<int64_t>(ATT_MIN_CHUNKS, (total + slots - 1) / slots);; per += per / 8 + 1) {
        a = AttnPlan4{b0, nb, (uint32_t)std::min<int64_t>(per, 1 << 27), 0, 0, 0, 0, 0};
        a.per_inv = (uint32_t)(((1ull << 32) + a.per - 1) / a.per);
        for (int b = b0; b < b0 + nb; ++b) {
            const Count4 c = count_items(h_lens[b], h_cu[b + 1] - h_cu[b], G, Hkv, p.rows_log2(), a.per, a.per_inv);
            a.n_items += c.items;
            a.n_records += c.records;
            a.n_merge_rows += c.merge_rows;
            a.swizzle |= c.tiles > 1;
        }
        if (p.wk != 8 || a.n_items <= slots || a.n_records == 0) break;
    }
}

}  // namespace

hipError_t launch_kv4_append(const Kv4Append &a, hipStream_t s) {
    // (workgroups for the chip to fill, as far as there are heads; each takes the token's angles anew)
    const int n_split = std::min((a.Hq + 2 * a.b.Hkv + 7) / 8, std::max(1, 1024 / a.b.T));
    kv4_append_kernel<<<(unsigned)a.b.T * n_split, 256, 0, s>>>(a, n_split);
    return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4Batch &b, float *k, float *v, hipStream_t s) {
    // (a workgroup for every eight heads, while a launch has less than 2^32 threads)
    const int n_split = std::min((b.Hkv + 7) / 8, std::max(1, ((1 << 24) - 1) / b.T));
    kv4_read_kernel<<<(unsigned)b.T * n_split, 256, 0, s>>>(b, n_split, k, v);
    return hipGetLastError();
}

namespace {
size_t part_o_bytes(const Launch4 &p) { return p.record_rows() * 128 * sizeof(float); }
size_t part_ml_bytes(const Launch4 &p) { return p.record_rows() * sizeof(float2); }
}  // namespace

size_t kv4_attn_scratch(const int32_t *h_cu, const int32_t *h_lens, int B, int Hq, int Hkv) {
    size_t need = 0;
    Launch4 p;
    for (int b0 = 0; b0 < B; b0 += ATT_TRACES) {      // (the launches follow one another: each may use all of it)
        plan_launch(p, h_cu, h_lens, b0, std::min(ATT_TRACES, B - b0), Hq, Hkv);
        need = std::max(need, part_o_bytes(p) + part_ml_bytes(p));
    }
    return need;
}

hipError_t launch_kv4_attn(const Kv4Attn &a, const int32_t *h_cu, const int32_t *h_lens, void *scratch, hipStream_t s) {
    Launch4 p;
    for (int b0 = 0; b0 < a.b.B; b0 += ATT_TRACES) {
        plan_launch(p, h_cu, h_lens, b0, std::min(ATT_TRACES, a.b.B - b0), a.Hq, a.b.Hkv);
        float *part_o = (float *)scratch;
        float2 *part_ml = (float2 *)((char *)scratch + part_o_bytes(p));
        const int threads = 64 * p.wr * p.wk;
        if (p.wr == 4) kv4_attn_kernel<2, 4, 1><<<p.plan.n_items, threads, 0, s>>>(a, p.plan, part_o, part_ml);
        else if (p.nq == 2 && p.wk == 8) kv4_attn_kernel<2, 1, 8><<<p.plan.n_items, threads, 0, s>>>(a, p.plan, part_o, part_ml);
        else if (p.nq == 2) kv4_attn_kernel<2, 1, 4><<<p.plan.n_items, threads, 0, s>>>(a, p.plan, part_o, part_ml);
        else if (p.wk == 4) kv4_attn_kernel<1, 1, 4><<<p.plan.n_items, threads, 0, s>>>(a, p.plan, part_o, part_ml);
        else kv4_attn_kernel<1, 1, 8><<<p.plan.n_items, threads, 0, s>>>(a, p.plan, part_o, part_ml);
        if (hipError_t e = hipGetLastError()) return e;
        if (p.plan.n_merge_rows) {
            kv4_merge_kernel<<<(p.plan.n_merge_rows + 3) / 4, 256, 0, s>>>(a, p.plan, p.rows_log2(), part_o, part_ml);
            if (hipError_t e = hipGetLastError()) return e;
        }
    }
    return hipSuccess;
}

}  // namespace cs
