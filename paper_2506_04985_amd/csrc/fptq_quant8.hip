// Activations to 8 bits with a scale for each token, for linears whose input four bits cannot carry: behind the residual's addition and an
// RMS norm (both optional), and behind the gated activation.
//
//   norm   z = x + r;  u = z * gain;  inv = 1 / sqrt(mean z^2 + eps)         gated   z = u = silu(gate) * up,  inv = 1
//   a = max |u|;  code = rne(u * (127 / a));  s_t = a * inv / 127
//
// The norm's factor is the same for a whole row, so it goes into the token's scale and not into the codes: one pass with one exchange between
// the waves of a row (a sum and a maximum at once), and a row's codes do not wait for a division and a root in 64 bits.  The row stays in registers
// from its load to its codes.  Bound: HBM, 2 to 4 bytes read and 1 to 3 written per value: norm with residual and gain 8192 x 8192 83 us, 5.65 TB/s (a copy of 2 GiB reaches 4.92), VALU busy in
// 40 % of the cycles; gated 4096 x 14336 58 us, 5.06 TB/s.  Few rows are a chain of latencies: launch, row, exchange, store (norm 1 x 4096 2.2 us in a kernel trace, gated 16 x 14336 6.3 to 6.7).
#include "fptq_common.h"

namespace fptq {

enum { PLAIN, RESIDUAL, GATED };

__device__ inline float low_f32(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ inline float high_f32(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

// silu(g) = g / (1 + e^-g), correct to the last bit of fp32 for every bf16 g, so that codes do not depend on whose exponential computed them: in 64 bits
// with about 2^-47 to spare.  e^-g = 2^n e^r, |r| <= ln 2 / 2, by its Taylor series to r^11 (r^12 / 12! < 2^-47); the quotient from the hardware's estimate by two
// Newton steps.  Beyond +-700 the exponential is that of 700: g or, in fp32, 0 (infinity stays infinite, NaN stays NaN).
__device__ inline float silu(float g)
{
    const double y = -(double)__builtin_amdgcn_fmed3f(g, -700.0f, 700.0f);
    const double n = __builtin_rint(y * 0x1.71547652b82fep+0), r = __builtin_fma(n, -0x1.62e42fefa39efp-1, y);
    double p = 1.0 / 39916800;
    p = __builtin_fma(p, r, 1.0 / 3628800);
    p = __builtin_fma(p, r, 1.0 / 362880);
    p = __builtin_fma(p, r, 1.0 / 40320);
    p = __builtin_fma(p, r, 1.0 / 5040);
    p = __builtin_fma(p, r, 1.0 / 720);
    p = __builtin_fma(p, r, 1.0 / 120);
    p = __builtin_fma(p, r, 1.0 / 24);
    p = __builtin_fma(p, r, 1.0 / 6);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    const double d = 1.0 + __builtin_ldexp(p, (int)n);
    double q = __builtin_amdgcn_rcp(d);
    q = __builtin_fma(q, __builtin_fma(-d, q, 1.0), q);
    q = __builtin_fma(q, __builtin_fma(-d, q, 1.0), q);
    return (float)((double)g * q);
}

// silu of the bf16 values of magnitude 2^-14 to 2^7, sign by sign in the order of their patterns: 21 KB of LDS, read once a workgroup, in place of 33 instructions a value, most of them in
// 64 bits, which bound the kernel (4096 x 14336 83 us).  That is for gates like those of a layer, of deviation 1.5; smaller ones fall below the table and are computed, a wave's chunk at a time: 4096 x 14336 56 us with
// deviation 1.5, 63 with 0.1, 84 with 0.02, 92 with zeros.  Made by the compiler with the same series, in 64 bits and rounded once.
constexpr int SILU_FIRST = (127 - 14) << 7, SILU_COUNT = 21 << 7;
struct SiluTable {
    float value[2 * SILU_COUNT];
};
static_assert(sizeof(SiluTable) % 1024 == 0, "whole wave loads");
constexpr SiluTable silu_table()
{
    SiluTable t = {};
    for (int i = 0; i < 2 * SILU_COUNT; ++i) {
        const double g = __builtin_bit_cast(float, (uint32_t)(SILU_FIRST + i % SILU_COUNT) << 16) * (i < SILU_COUNT ? 1.0 : -1.0);
        const double m = -g * 0x1.71547652b82fep+0;
        const int n = (int)(m < 0 ? m - 0.5 : m + 0.5);
        const double r = (-g - n * 0x1.62e42fep-1) - n * 0x1.f473de6af278fp-30;      // ln 2 in two pieces, n times the first exact
        double p = 1.0;
        for (int k = 14; k > 0; --k) p = 1.0 + p * r / k;
        t.value[i] = (float)(g / (1.0 + p * __builtin_bit_cast(double, (uint64_t)(1023 + n) << 52)));
    }
    return t;
}
__device__ const SiluTable SILU = silu_table();

// What a row's maximum of |u|, as bits, says: NaN and infinities are the largest patterns, so a row that holds one is told by its maximum.
struct Grid {
    uint32_t largest;
    float a, step;          // u * step is a code
    bool finite;
    __device__ Grid(uint32_t bits) : largest(bits), finite(bits < 0x7f800000u)
    {
        a = fmaxf(__uint_as_float(bits), 0x1p-100f);      // below, 127 / a would not be finite
        step = 127.0f / a;
    }
    // 0 for a row of zeros, also where its factor is infinite (eps = 0); NaN where a value is not finite, so that no output of the token looks like one
    __device__ float token_scale(float inv) const
    {
        return !finite ? __uint_as_float(0x7fc00000u) : largest == 0u ? 0.0f : a * inv * (1.0f / 127.0f);
    }
};

// Codes of eight values in the order of the layout.  1.5 * 2^23 is added to a product, whose sum holds the rounded integer in its low byte.
__device__ inline uint2 codes_of(const float (&u)[8], const Grid &g)
{
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(u[e] * g.step + 12582912.0f);
    auto join = [&](int i) {      // the low bytes of b[i], b[i + 2], b[i + 4], b[i + 6]
        const uint32_t lo = __builtin_amdgcn_perm(b[i + 2], b[i], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[i + 6], b[i + 4], 0x04000c0cu);
        return lo | hi;
    };
    return g.finite ? make_uint2(join(0), join(1)) : make_uint2(0u, 0u);
}

// silu(gate) * up of eight values by the table, two 16-bit places of it in a register; where any lane's gate lies outside it (`live` lanes: the others hold zeros) the chunk is computed.
typedef unsigned short v2us __attribute__((ext_vector_type(2)));
__device__ inline void gated_eight(const uint32_t (&aw)[4], const uint32_t (&bw)[4], bool live, const float *table, float (&z)[8])
{
    v2us far = {0, 0};
    uint32_t at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const v2us a = __builtin_bit_cast(v2us, aw[j] & 0x7fff7fffu) - (v2us){SILU_FIRST, SILU_FIRST}, sign = __builtin_bit_cast(v2us, aw[j]) >> 15;
        far = __builtin_elementwise_max(far, a);
        at[j] = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(a, (v2us){SILU_COUNT - 1, SILU_COUNT - 1}) + sign * (unsigned short)SILU_COUNT);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) z[2 * j] = table[at[j] & 0xffffu], z[2 * j + 1] = table[at[j] >> 16];
    if (__any(live && max(far.x, far.y) >= SILU_COUNT)) {
#pragma unroll 1
        for (int j = 0; j < 4; ++j) {      // rolled: gates of zero and beyond the table are taken to be few
            const float s0 = silu(low_f32(aw[j])), s1 = silu(high_f32(aw[j]));
            if (j == 0) z[0] = s0, z[1] = s1;
            if (j == 1) z[2] = s0, z[3] = s1;
            if (j == 2) z[4] = s0, z[5] = s1;
            if (j == 3) z[6] = s0, z[7] = s1;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) z[2 * j] *= low_f32(bw[j]), z[2 * j + 1] *= high_f32(bw[j]);
}

// z of eight values, and their squares
template <int KIND, bool TABLE>
__device__ inline void eight(const v4u &a, const v4u &b, bool live, const float *table, float (&z)[8], double &ss)
{
    const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
    if (KIND == GATED && TABLE) {
        gated_eight(aw, bw, live, table, z);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float z0 = low_f32(aw[j]), z1 = high_f32(aw[j]);
        if (KIND == GATED) z0 = silu(z0) * low_f32(bw[j]), z1 = silu(z1) * high_f32(bw[j]);
        if (KIND == RESIDUAL) z0 += low_f32(bw[j]), z1 += high_f32(bw[j]);
        if (KIND != GATED) {
            ss = add_square(ss, z0);
            ss = add_square(ss, z1);
        }
        z[2 * j] = z0, z[2 * j + 1] = z1;
    }
}

__device__ inline void multiply(float (&u)[8], const v4u &gain)
{
    const uint32_t w[4] = {gain.x, gain.y, gain.z, gain.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) u[2 * j] *= low_f32(w[j]), u[2 * j + 1] *= high_f32(w[j]);
}

__device__ inline v4u to_bf16(const float (&z)[8]) { return v4u{pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]), pack_bf16(z[4], z[5]), pack_bf16(z[6], z[7])}; }

__device__ inline uint32_t largest_of(uint32_t m, const float (&u)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(u[e]) & 0x7fffffffu);
    return m;
}

__device__ inline float inverse_rms(double ss, double K, float eps, int rms) { return rms ? (float)(1.0 / sqrt(ss / K + (double)eps)) : 1.0f; }

// WPR waves take a row (1: four rows a workgroup, no LDS and no barrier), CH chunks of eight values a lane.  Aligned rows are read through row-sized
// descriptors (chunks past the end are zero); RAGGED: chunks of any alignment, where they lie.  The new residual may be the buffer of either input: all loads of a row come
// before its maximum is known, and that before its first store.  A workgroup goes on from row to row where there are more than a launch may hold,
// and, with the table, where there are more rows than workgroups that the device runs at once: the next row's loads are then issued as soon as this one's values are made.
template <int KIND, int WPR, int CH, bool RAGGED, bool TABLE>
__global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR) void quantize8_kernel(const uint16_t *a, const uint16_t *b, uint8_t *__restrict__ out, float *__restrict__ scale,
                                                                              int K, int rows, const uint16_t *__restrict__ gain, int64_t a_stride, int64_t b_stride,
                                                                              uint16_t *sum_out, float eps, int rms)
{
    constexpr int S = 64 * WPR;
    constexpr bool KEEP = KIND == GATED || WPR * CH < 48;      // else u is made of z a second time, with the gain read again: registers for u and the new residual do not suffice
    __shared__ double red_sum[2][WPR > 1 ? WPR : 1];
    __shared__ uint32_t red_max[2][WPR > 1 ? WPR : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = WPR == 1 ? lane : (int)threadIdx.x, padded = (K + KT - 1) / KT * KT;
    const int64_t M = rows;
    const int64_t t0 = WPR == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x, t_step = (int64_t)gridDim.x * (WPR == 1 ? 4 : 1);
    v4u av[CH], bv[CH], gv[CH], sums[CH];
    auto load = [&](int64_t t) {
        const uint16_t *const arow = a + t * a_stride, *const brow = KIND == PLAIN ? arow : b + t * b_stride;
        if (RAGGED) {
            load_row_chunks(av, arow, h * 8, S * 8, K);
            if (KIND != PLAIN) load_row_chunks(bv, brow, h * 8, S * 8, K);
        } else {
            const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc((void *)arow, 0, K * 2, RSRC_FLAGS);
            const __amdgpu_buffer_rsrc_t br = __builtin_amdgcn_make_buffer_rsrc((void *)brow, 0, K * 2, RSRC_FLAGS);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                av[i] = __builtin_amdgcn_raw_buffer_load_b128(ar, (i * S + h) * 16, 0, 0);
                if (KIND != PLAIN) bv[i] = __builtin_amdgcn_raw_buffer_load_b128(br, (i * S + h) * 16, 0, 0);
            }
        }
    };
    __shared__ __attribute__((aligned(1024))) float table[TABLE ? 2 * SILU_COUNT : 4];
    if (TABLE) {      // on its way to LDS while the first row is to the registers
        const __amdgpu_buffer_rsrc_t tr = __builtin_amdgcn_make_buffer_rsrc((void *)SILU.value, 0, (int)sizeof SILU, RSRC_FLAGS);
        for (int i = wave; i < (int)sizeof SILU / 1024; i += WPR == 1 ? 4 : WPR)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(tr, LDS_PTR(reinterpret_cast<uint8_t *>(table) + i * 1024), 16, i * 1024 + lane * 16, 0, 0, 0);
        if (t0 < M) load(t0);
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        __syncthreads();
    }
    int turn = 0;
    for (int64_t t = t0; t < M; t += t_step, turn ^= 1) {
        if (!TABLE) load(t);
        if (KEEP && KIND != GATED && gain) {
            if (RAGGED) {
                load_row_chunks(gv, gain, h * 8, S * 8, K);
            } else {
                const __amdgpu_buffer_rsrc_t gr = __builtin_amdgcn_make_buffer_rsrc((void *)gain, 0, K * 2, RSRC_FLAGS);
#pragma unroll
                for (int i = 0; i < CH; ++i) gv[i] = __builtin_amdgcn_raw_buffer_load_b128(gr, (i * S + h) * 16, 0, 0);
            }
        }
        float u[CH][8];
        double ss = 0.0;
        uint32_t largest = 0;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            eight<KIND, TABLE>(av[i], bv[i], (i * S + h) * 8 < K, table, u[i], ss);
            if (KIND == RESIDUAL && KEEP) sums[i] = to_bf16(u[i]);
            if (KEEP) {
                if (KIND != GATED && gain) multiply(u[i], gv[i]);
                largest = largest_of(largest, u[i]);
            } else {
                float scaled[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) scaled[e] = u[i][e];
                if (gain) {
                    v4u now[1];
                    load_row_chunks(now, gain, (i * S + h) * 8, 0, K);
                    multiply(scaled, now[0]);
                }
                largest = largest_of(largest, scaled);
            }
        }
        if (TABLE && t + t_step < M) load(t + t_step);
        largest = wave_max(largest);
        if (KIND != GATED && rms) ss = wave_sum(ss);
        if (WPR > 1) {
            if (lane == 0) red_max[turn][wave] = largest, red_sum[turn][wave] = ss;
            __syncthreads();
            largest = 0;
#pragma unroll
            for (int w = 0; w < WPR; ++w) largest = max(largest, red_max[turn][w]);
        }
        const Grid grid(largest);
        if (h == 0) {      // the others go on
            if (WPR > 1 && KIND != GATED && rms) {
                ss = 0.0;
                for (int w = 0; w < WPR; ++w) ss += red_sum[turn][w];
            }
            scale[t] = grid.token_scale(KIND == GATED ? 1.0f : inverse_rms(ss, (double)K, eps, rms));
        }
        uint8_t *const at = out + (((int64_t)(h >> 4) * M + t) * KT + (h & 15) * 8);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int k0 = (i * S + h) * 8;
            if (!KEEP) {
                if (KIND == RESIDUAL) sums[i] = to_bf16(u[i]);
                if (gain) {
                    v4u again[1];
                    load_row_chunks(again, gain, k0, 0, K);
                    multiply(u[i], again[0]);
                }
            }
            if (k0 < padded) *reinterpret_cast<uint2 *>(at + (int64_t)(S / 16 * i) * M * KT) = codes_of(u[i], grid);      // padding is zero like its input
            if (KIND == RESIDUAL && sum_out) {
                uint16_t *const to = sum_out + t * (int64_t)K + k0;
                if (!RAGGED) {
                    if (k0 < K) *reinterpret_cast<v4u *>(to) = sums[i];
                } else if (k0 + 8 <= K) {
                    __builtin_memcpy(to, &sums[i], 16);
                } else {
                    const uint32_t w[4] = {sums[i].x, sums[i].y, sums[i].z, sums[i].w};
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (k0 + e < K) to[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                }
            }
        }
    }
}

// Rows that the registers do not hold: a workgroup reads a row twice, the second time from the caches.  A thread stores only what no other one reads.
template <int KIND>
__global__ __launch_bounds__(1024) void quantize8_long_kernel(const uint16_t *a, const uint16_t *b, uint8_t *__restrict__ out, float *__restrict__ scale, int64_t K,
                                                              int64_t M, const uint16_t *__restrict__ gain, int64_t a_stride, int64_t b_stride, uint16_t *sum_out,
                                                              float eps, int rms)
{
    __shared__ double red_sum[16];
    __shared__ uint32_t red_max[16];
    for (int64_t t = blockIdx.x; t < M; t += gridDim.x) {
        const uint16_t *arow = a + t * a_stride, *brow = KIND == PLAIN ? arow : b + t * b_stride;
        auto f = [](uint16_t v) { return __uint_as_float((uint32_t)v << 16); };
        auto value = [&](int64_t k) { return KIND == GATED ? silu(f(arow[k])) * f(brow[k]) : KIND == RESIDUAL ? f(arow[k]) + f(brow[k]) : f(arow[k]); };
        double ss = 0.0;
        uint32_t largest = 0;
        for (int64_t k = threadIdx.x; k < K; k += 1024) {
            const float z = value(k), u = gain ? z * f(gain[k]) : z;
            ss = add_square(ss, z);
            largest = max(largest, __float_as_uint(u) & 0x7fffffffu);
        }
        largest = wave_max(largest);
        ss = wave_sum(ss);
        if ((threadIdx.x & 63) == 0) red_max[threadIdx.x >> 6] = largest, red_sum[threadIdx.x >> 6] = ss;
        __syncthreads();
        largest = 0, ss = 0.0;
        for (int w = 0; w < 16; ++w) largest = max(largest, red_max[w]), ss += red_sum[w];
        __syncthreads();
        const Grid grid(largest);
        if (threadIdx.x == 0) scale[t] = grid.token_scale(KIND == GATED ? 1.0f : inverse_rms(ss, (double)K, eps, rms));
        const int64_t padded = k_tiles(K) * KT;
        for (int64_t k0 = (int64_t)threadIdx.x * 8; k0 < padded; k0 += 8192) {
            float u[8];
            for (int e = 0; e < 8; ++e) {
                const int64_t k = k0 + e;
                u[e] = 0.0f;
                if (k < K) {
                    const float z = value(k);
                    u[e] = gain ? z * f(gain[k]) : z;
                    if (KIND == RESIDUAL && sum_out) sum_out[t * K + k] = (uint16_t)(pack_bf16(z, 0.0f) & 0xffffu);
                }
            }
            *reinterpret_cast<uint2 *>(out + ((k0 / KT) * M + t) * KT + k0 % KT) = codes_of(u, grid);
        }
    }
}

// Library layout -> one int8 per value, row-major (checking only).
__global__ __launch_bounds__(256) void unpack8_kernel(const uint8_t *__restrict__ packed, int64_t rows, int64_t K, int8_t *__restrict__ out)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * K; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / K, k = i % K;
        out[i] = (int8_t)packed[((k / KT) * rows + row) * KT + (k % KT) / 8 * 8 + (k % 2) * 4 + k % 8 / 2];
    }
}

hipError_t launch_unpack8(const uint8_t *packed, int64_t rows, int64_t K, int8_t *out, hipStream_t s)
{
    const int64_t blocks = (rows * K + 255) / 256;
    unpack8_kernel<<<dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), 0, s>>>(packed, rows, K, out);
    return hipGetLastError();
}

constexpr int64_t MOST_WORKGROUPS = (int64_t)1 << 20;      // of a launch, whose threads have to stay below 2^32

// Workgroups of the gated kernel with the table that a CU runs at once, by the table's LDS (7), a SIMD's eight waves (seven for ragged rows, whose kernels take more than 100 scalar registers), or
// from three chunks a lane on the vector registers.
template <int WPR, int CH, bool RAGGED>
constexpr int resident()
{
    if (WPR <= 4) return CH <= 2 ? 7 : 5;
    if (WPR == 8) return CH == 4 ? 2 : (CH == 3 ? 3 : 4) - RAGGED;
    return CH <= 2 && !RAGGED ? 2 : 1;
}

template <int KIND, int WPR, int CH, bool TABLE>
static hipError_t launch_rows(bool vec, const uint16_t *a, const uint16_t *b, const uint16_t *gain, int64_t M, int64_t K, int64_t a_stride, int64_t b_stride, int rms,
                              float eps, uint8_t *out, float *scale, uint16_t *sum_out, hipStream_t s)
{
    int64_t blocks = WPR == 1 ? (M + 3) / 4 : M;
    if (TABLE) {      // a workgroup reads the table once and goes on from row to row: as many as fit the device together, and where a CU holds one, as many as come to the same number of rows each
        // (on 1100 sizes: so 4 % faster than with the same number of rows each where a CU holds several, 1 % slower where it holds one; 600 x 28001 34.0 us with two workgroups a CU asked for, 26.5 with the one it holds)
        const int64_t cus = device_cus_or_default(), a_cu = vec ? resident<WPR, CH, false>() : resident<WPR, CH, true>(), room = cus * a_cu, each = (blocks + room - 1) / room;
        blocks = a_cu == 1 ? (blocks + each - 1) / each : blocks < room ? blocks : room;
    }
    const dim3 grid((unsigned)(blocks < MOST_WORKGROUPS ? blocks : MOST_WORKGROUPS)), block(WPR == 1 ? 256 : 64 * WPR);
    if (vec)
        quantize8_kernel<KIND, WPR, CH, false, TABLE><<<grid, block, 0, s>>>(a, b, out, scale, (int)K, (int)M, gain, a_stride, b_stride, sum_out, eps, rms);
    else
        quantize8_kernel<KIND, WPR, CH, true, TABLE><<<grid, block, 0, s>>>(a, b, out, scale, (int)K, (int)M, gain, a_stride, b_stride, sum_out, eps, rms);
    return hipGetLastError();
}

template <int KIND>
static hipError_t launch(const uint16_t *a, const uint16_t *b, const uint16_t *gain, int64_t M, int64_t K, int64_t a_stride, int64_t b_stride, int rms, float eps,
                         uint8_t *out, float *scale, uint16_t *sum_out, hipStream_t s)
{
    auto aligned = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const bool vec = K % 8 == 0 && aligned(a) && aligned(b) && aligned(gain) && aligned(sum_out) && a_stride % 8 == 0 && b_stride % 8 == 0;
    // As many threads as the row has chunks, two or three chunks each where that is more than 512, on 17078 sizes measured with data in no cache (rows / workgroup): the rule is within 1 % of the
    // best of 22 shapes on average, 3 to 7 % at the 95th percentile (gated rows on 30593 sizes: beyond 4096 values 0 to 3 % on average, in shorter ones up to 5 % with 2048 rows, 0 to 22 % with more, where a
    // wave or two a row with three or four chunks a lane would do better).  us, norm with residual, rows of 7391 values / 8192 / 14336: 333 x 16 waves of one chunk 9.5, 8 of two 7.6; 8192 x 97.6 and 92.2;
    // 4096 x 16 of two 91.3, 8 of four 95.0.  The gated kernel reads its table where there are enough values to a workgroup: 4096 x 14336 83.6 without, 55.6 with it, 32 x 4096 3.4 and 4.2.
#define FPTQ_ROWS(WPR, CH, TABLE) return launch_rows<KIND, WPR, CH, TABLE && KIND == GATED>(vec, a, b, gain, M, K, a_stride, b_stride, rms, eps, out, scale, sum_out, s)
    if (M <= 0x7fffffff && K <= 32768) {
        constexpr bool G = KIND == GATED;
        if (K <= 4096 && !(G && M * K > 3 << 19)) {
            if (K <= 512) FPTQ_ROWS(1, 1, false);
            if (K <= 1024 && M <= 2048) FPTQ_ROWS(2, 1, false);
            if (K <= 1024) FPTQ_ROWS(1, 2, false);
            if (K <= 2048 && M <= 2048) FPTQ_ROWS(4, 1, false);
            if (K <= 2048) FPTQ_ROWS(2, 2, false);
            if (M <= 1024) FPTQ_ROWS(8, 1, false);
            FPTQ_ROWS(4, 2, false);
        }
        if constexpr (G) {
            if (K <= 512) FPTQ_ROWS(1, 1, true);
            if (K <= 1024) FPTQ_ROWS(1, 2, true);
            if (K <= 2048) FPTQ_ROWS(4, 1, true);
            if (K <= 4096 && M <= 1024) FPTQ_ROWS(8, 1, true);
            if (K <= 4096) FPTQ_ROWS(4, 2, true);
            if (K <= 8192 && M <= 256) FPTQ_ROWS(16, 1, true);
            if (K <= 8192 && M <= 1024) FPTQ_ROWS(8, 2, true);
            if (K > 12288 && K <= 16384 && M > 256) FPTQ_ROWS(8, 4, true);
        }
        if (K <= 6144) FPTQ_ROWS(4, 3, true);
        if (K <= 8192) FPTQ_ROWS(8, 2, true);
        if (K <= 12288) FPTQ_ROWS(8, 3, true);
        if (K <= 16384) FPTQ_ROWS(16, 2, true);
        if (K <= 24576) FPTQ_ROWS(16, 3, true);
        FPTQ_ROWS(16, 4, true);
    }
#undef FPTQ_ROWS
    quantize8_long_kernel<KIND><<<dim3((unsigned)(M < MOST_WORKGROUPS ? M : MOST_WORKGROUPS)), dim3(1024), 0, s>>>(a, b, out, scale, K, M, gain, a_stride, b_stride, sum_out, eps,
                                                                                                                   rms);
    return hipGetLastError();
}

hipError_t launch_norm_quantize8(const uint16_t *x, const uint16_t *residual, const uint16_t *gain, int64_t M, int64_t K, int rms, float eps, uint8_t *out, float *scale,
                                 uint16_t *residual_out, hipStream_t s)
{
    return residual ? launch<RESIDUAL>(x, residual, gain, M, K, K, K, rms, eps, out, scale, residual_out, s)
                    : launch<PLAIN>(x, nullptr, gain, M, K, K, 0, rms, eps, out, scale, nullptr, s);
}

hipError_t launch_gated_quantize8(const uint16_t *gate, const uint16_t *up, int64_t M, int64_t K, int64_t gate_stride, int64_t up_stride, uint8_t *out, float *scale,
                                  hipStream_t s)
{
    return launch<GATED>(gate, up, nullptr, M, K, gate_stride, up_stride, 0, 0.0f, out, scale, nullptr, s);
}

}  // namespace fptq
