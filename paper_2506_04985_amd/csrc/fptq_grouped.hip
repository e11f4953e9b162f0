// Linear layer of 8-bit activations and packed 4-bit weights with a scale for each group of K values:
//     y[t, n] = s_t * sum_g s[g, n] * (sum over k in g of code[t, k] * w[n, k])
// The inner sum is an integer and exact; those of the groups are added in fp32.
//
// Nibbles are widened to bytes that hold 16 * value as in the other linears, (p << 4) & 0xF0F0F0F0 and p & 0xF0F0F0F0, and the codes of eight k lie
// in that order, so they are operands as they are.  Of 128 k or fewer, 16 * sum stays below 2^21 in magnitude, which fp32 holds exactly; the 1/16 goes into the
// output, exactly as well.  Groups of several K tiles take their scale once a tile.
#include <utility>

#include "fptq_common.h"

namespace fptq {

typedef int v2i __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));

__device__ inline v2i widen1(int p) { return v2i{(p << 4) & (int)0xF0F0F0F0, p & (int)0xF0F0F0F0}; }
__device__ inline v4i widen2(int p0, int p1)
{
    const v2i a = widen1(p0), b = widen1(p1);
    return v4i{a.x, a.y, b.x, b.y};
}

// What a lane of a few-token wave holds of a K tile.  Weights: lane (c = l % 16, q = l / 16) loads granule q (16 bytes: k = 32 q ...) of channel c, so a
// wave's load is 1 KB in one piece.  The MFMAs must not mix groups, so where a tile holds several, lanes exchange dwords: two groups by swapping halves of
// the wave, four by a 4 x 4 transposition between its quarters.  GT: groups a tile.
template <int GT>
__device__ inline void by_group(v4i &w)
{
    if (GT == 1) return;
    auto swap32 = [](int &a, int &b) {
        const auto r = __builtin_amdgcn_permlane32_swap((uint32_t)a, (uint32_t)b, false, false);
        a = (int)r[0], b = (int)r[1];
    };
    auto swap16 = [](int &a, int &b) {
        const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)a, (uint32_t)b, false, false);
        a = (int)r[0], b = (int)r[1];
    };
    int d0 = w.x, d1 = w.y, d2 = w.z, d3 = w.w;
    swap32(d0, d2), swap32(d1, d3);                    // dwords 0 and 1: lanes' k below 64 (of lanes q and q - 2), 2 and 3: above
    if (GT == 4) swap16(d0, d1), swap16(d2, d3);
    w = v4i{d0, d1, d2, d3};
}

// An output of a sum of 16 * value: the 1/16 goes where it loses nothing, into the token's scale, or into the sum where the scale's lowest bits would fall out of fp32's subnormal range (a sum
// that loses bits then comes to zero in any case).
struct OutputScale {
    float of_sum, of_token;
    __device__ explicit OutputScale(float s) : of_sum(fabsf(s) < 0x1p-122f ? 0.0625f : 1.0f), of_token(fabsf(s) < 0x1p-122f ? s : s * 0.0625f) {}
    template <class T>
    __device__ T operator()(T sum) const
    {
        return sum * of_sum * of_token;
    }
};

// Few tokens.  A workgroup owns 16 RT channels of 16 tokens, its waves split K (wave w takes K tiles w, w + WAVES, ...) with one K tile in flight each and
// several workgroups a CU.  Bound: HBM, the weights once, streamed, up to 16 tokens; of more tokens every 16 load, widen and reorder all weights again (1 x 4096 x 4096 4.1 us,
// 16 x 5.1, 32 x 6.1).  Tokens are the rows of the MFMA's result and channels its columns, so that a lane has one channel, and
// one scale of it a group.  The waves' fp32 sums meet in LDS and are added in order.
template <int WAVES, int RT, int GT>
__global__ __launch_bounds__(64 * WAVES) void grouped_few_kernel(const uint8_t *__restrict__ x, const uint8_t *__restrict__ w, const float *__restrict__ scales, int M,
                                                                 int N, int ktiles, int groups, uint32_t tiles_per_group, uint32_t reciprocal_of_it,
                                                                 const float *__restrict__ token_scale, void *__restrict__ y, int y_type)
{
    __shared__ float red[WAVES][RT * 256];
    static_assert(RT * 256 <= 64 * WAVES, "an output a thread");
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = blockIdx.x * (16 * RT), m0 = blockIdx.y * 16;
    const int64_t w_slab = (int64_t)N * SEG, x_slab = (int64_t)M * KT;
    const uint8_t *wp[RT];
    const float *sp[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int n = min(n0 + rt * 16 + c, N - 1);      // channels and tokens past the end repeat the last one; what they make is not stored
        wp[rt] = w + (int64_t)n * SEG + q * 16;
        sp[rt] = scales + n;
    }
    // a token's 16 or 8 codes for each MFMA, as by_group leaves the weights
    constexpr int STEPS = GT == 4 ? 4 : 2, X_STEP = GT == 1 ? 16 : GT == 2 ? 64 : 32;
    const int x_first = GT == 1 ? q * 32 : GT == 2 ? (q & 1) * 32 + (q >> 1) * 16 : q * 8;
    const uint8_t *const xp = x + (int64_t)min(m0 + c, M - 1) * KT + x_first;
    // what the thread's output will need, fetched now: the kernel is too short to end on a memory latency
    const int t_out = m0 + tid / (16 * RT), n_out = n0 + tid % (16 * RT);
    const bool stores = tid < RT * 256 && t_out < M && n_out < N;
    const OutputScale scaled(stores ? token_scale[t_out] : 0.0f);

    v4f sum[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) sum[rt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int kt = wave; kt < ktiles; kt += WAVES) {
        v4i wv[RT], xv[STEPS];
        float sv[RT][GT];
        uint32_t first, rest;
        divide((uint32_t)kt, tiles_per_group, reciprocal_of_it, first, rest);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            wv[rt] = __builtin_nontemporal_load(reinterpret_cast<const v4i *>(wp[rt] + kt * w_slab));
#pragma unroll
            for (int g = 0; g < GT; ++g) sv[rt][g] = sp[rt][(int64_t)min((int)first * GT + g, groups - 1) * N];      // a last tile may hold fewer groups: its weights there are zero
        }
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            if (GT == 4) {
                const v2i v = *reinterpret_cast<const v2i *>(xp + kt * x_slab + j * X_STEP);
                xv[j] = v4i{v.x, v.y, 0, 0};
            } else {
                xv[j] = *reinterpret_cast<const v4i *>(xp + kt * x_slab + j * X_STEP);
            }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            by_group<GT>(wv[rt]);
            v4i acc = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < STEPS; ++j) {
                if constexpr (GT == 4)
                    acc = __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, v2i{xv[j].x, xv[j].y}), __builtin_bit_cast(long, widen1(wv[rt][j])), v4i{0, 0, 0, 0}, 0, 0, 0);
                else
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(xv[j], widen2(wv[rt][2 * j], wv[rt][2 * j + 1]), GT == 2 ? v4i{0, 0, 0, 0} : acc, 0, 0, 0);
                if (GT != 1 || j == 1) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[rt][r] = __builtin_fmaf((float)acc[r], sv[rt][GT == 1 ? 0 : j], sum[rt][r]);
                }
            }
        }
    }

    // lane l, register r holds token 4 (l / 16) + r, channel l % 16
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[wave][(4 * q + r) * (16 * RT) + rt * 16 + c] = sum[rt][r];
    __syncthreads();
    if (!stores) return;
    float v = red[0][tid];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v += red[i][tid];
    v = scaled(v);
    if (y_type == FPTQ_F32)
        static_cast<float *>(y)[(int64_t)t_out * N + n_out] = v;
    else
        static_cast<uint16_t *>(y)[(int64_t)t_out * N + n_out] = bf16_rne(v);
}

// y's four channels from n on of token t, from sums of 16 * value.  Streamed stores: 4096 x 28672 x 1024 166.5 us, 161 with them, 333 x 32003 x 2504 42.8 and 42.1; the gated quantizer behind
// them reads as fast (512 x 28672 x 4096 with it 83.8 and 81.3, 4096 x 28672 x 4096 549 and 550).
typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef v2u v2u_anywhere __attribute__((aligned(2)));
typedef v4f v4f_anywhere __attribute__((aligned(4)));
constexpr int PARTIAL = 2;      // beside FPTQ_BF16 and FPTQ_F32: the sums as they are
__device__ inline void store_four(v4f v, float scale, int t, int n, int N, void *y, int y_type)
{
    v = OutputScale(scale)(v);
    if (y_type == FPTQ_F32) {
        float *const to = static_cast<float *>(y) + (int64_t)t * N + n;
        if (n + 4 <= N) {
            __builtin_nontemporal_store((v4f_anywhere)v, reinterpret_cast<v4f_anywhere *>(to));
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (n + e < N) to[e] = v[e];
        }
    } else {
        uint16_t *const to = static_cast<uint16_t *>(y) + (int64_t)t * N + n;
        const uint32_t pair[2] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        if (n + 4 <= N) {
            __builtin_nontemporal_store((v2u_anywhere){pair[0], pair[1]}, reinterpret_cast<v2u_anywhere *>(to));
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (n + e < N) to[e] = (uint16_t)(pair[e / 2] >> (16 * (e % 2)));
        }
    }
}

// ---- tiles, for more tokens than a few
//
// A workgroup makes BN channels x BM tokens, each of its waves TN x TM sub-tiles of 32 x 32.  A K tile of both operands and its groups' scales go from HBM to LDS
// by loads that write LDS directly, STAGES deep, one barrier a K tile.  v_mfma_i32_32x32x32_i8 makes a group's integer sums, which go into the fp32 sums at once: with tokens
// as rows of the result and channels as columns a lane has one channel of a sub-tile, so its scale is one register, and (float)sum and a fused multiply-add are the 32
// vector instructions that the 4 MFMAs of a 128-value group cost.  KS sets of WAVES waves share the tile, set g taking K tiles g, g + KS, ... through a ring of its own; with one wave in a set
// nobody waits for another before the end.
//
// What bounds the large tiles: those conversions beside the MFMAs, then power.  An MFMA takes 33.5 cycles alone, with four conversions and four multiply-adds behind it 51, with eight multiply-adds 47.6 (two waves a
// SIMD, measured in registers); 256 x 256 walks a K tile in 1.50 us on zeros, 56 cycles an MFMA, and in 1.9 on dense operands, where the clock falls to 1.75 GHz (4096 x 28672 x 4096 464 to 497 us, 1.9 to
// 2.1 POP/s; MFMAs busy in 47 % of the cycles).  Two waves a SIMD, so that one's conversions run under the other's MFMAs; within a wave they are pinned behind the MFMAs of the next
// unit, without which that launch took 539 us on a card where it now takes 514.
//
// The MFMAs start from 0x4b400000, the pattern of the float 1.5 * 2^23: a sum below 2^22 (128 terms of at most 127 * 128 come to 2^21) is added to its low bits, and the result, taken as a float, less
// 1.5 * 2^23 is the sum exactly.  The subtraction issues at twice the conversion's rate: 2048 x 28672 x 4096 with groups of 32 491 us with conversions, 475 so; 1000 x 4096 x 14336 on 256 x 192 with
// groups of 64 199 and 191; 4096 x 28672 x 4096 504 and 496.
typedef int v16i __attribute__((ext_vector_type(16)));

template <int WAVES_N_, int WAVES_M_, int TN_, int TM_, int STAGES_, int KS_, int GT_>
struct Tile {
    static constexpr int WAVES_N = WAVES_N_, WAVES_M = WAVES_M_, TN = TN_, TM = TM_, STAGES = STAGES_, KS = KS_, GT = GT_;
    static constexpr int BN = WAVES_N * TN * 32, BM = WAVES_M * TM * 32, WAVES = WAVES_N * WAVES_M, THREADS = 64 * WAVES * KS;
    static constexpr int X_BYTES = BM * KT, W_BYTES = BN * SEG, S_BYTES = BN * GT * 4, STAGE_BYTES = X_BYTES + W_BYTES + S_BYTES;
    static constexpr int X_LOADS = X_BYTES / (WAVES * 1024), W_LOADS = W_BYTES / (WAVES * 1024), S_PIECES = BN * GT / 64, S_LOADS = (S_PIECES + WAVES - 1) / WAVES;
    static constexpr int LOADS = X_LOADS + W_LOADS + S_LOADS, RING_BYTES = STAGES * STAGE_BYTES;
    static constexpr int SETS = TN * TM * 16 <= 96 && TM > 1 && TN * TM * GT < 24 ? 2 : 1;
    static constexpr bool PRESET = TN * TM < 8 || GT == 1;      // where the constants' 16 registers do not spill
    static constexpr int OUT_ROWS = WAVES_M * 32, OUT_BYTES = KS * OUT_ROWS * BN * 4;      // a pass of the epilogue
    static constexpr int PASSES = TM > 1 && 2 * OUT_BYTES <= KS * RING_BYTES ? 2 : 1;      // of them that LDS holds
    static constexpr int SCALES_AT = KS * RING_BYTES > OUT_BYTES ? KS * RING_BYTES : OUT_BYTES, LDS_BYTES = SCALES_AT + BM * 4;      // the tokens' scales lie behind
    static constexpr int TOKEN_PIECES = (BM + 63) / 64;      // loads that bring them, a wave each
    static constexpr __host__ __device__ bool loads_token(int piece, int lane) { return BM % 64 == 0 || piece * 64 + lane < BM; }      // a last piece may be half a wave
    static_assert(X_BYTES % (WAVES * 1024) == 0 && W_BYTES % (WAVES * 1024) == 0 && BN % 64 == 0, "a K tile is shared out evenly");
    static_assert(S_PIECES % WAVES == 0 || WAVES % S_PIECES == 0, "waves without a piece of their own repeat another's");
    static_assert(LOADS * (STAGES - 1) < 64, "the count of loads in flight has six bits");
    static_assert(LDS_BYTES <= 160 * 1024 && OUT_ROWS * BN / 4 % THREADS == 0, "");
};

// where a K tile comes from and goes to
struct Fill {
    __amdgpu_buffer_rsrc_t x, w;
    uint8_t *base;
    int first, live;      // its first group; whether it is one
};

template <class F, int... I>
__device__ inline void in_order(std::integer_sequence<int, I...>, F f)
{
    (f(std::integral_constant<int, I>()), ...);
}

template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void grouped_tile_kernel(const uint8_t *__restrict__ x, const uint8_t *__restrict__ w, const float *__restrict__ scales, int M, int N,
                                                                     int ktiles, int tiles_m, int tiles_n, uint32_t tiles_per_group, uint32_t reciprocal_of_it, int groups,
                                                                     const float *__restrict__ token_scale, void *__restrict__ y, int y_type, int split_tiles)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave_all = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = C::KS > 1 ? wave_all / C::WAVES : 0, wave = C::KS > 1 ? wave_all % C::WAVES : wave_all;
    const int wave_n = wave % C::WAVES_N, wave_m = wave / C::WAVES_N, i32 = lane & 31, h = lane >> 5;
    uint8_t *const ring = lds + kg * C::RING_BYTES;

    // Workgroups go round the 8 XCDs; each gets a contiguous run of tiles, in bands of 8 along n, so that tiles that run together share operands in its L2.
    // y_type PARTIAL: workgroup (split, tile), tiles fastest, takes K tiles split_tiles * split ... and leaves its sums in y as fp32 [splits][M][N rounded up to 4].
    const int total = tiles_m * tiles_n, split = y_type == PARTIAL ? (int)blockIdx.x / total : 0, kt0 = split * split_tiles, kt1 = min(ktiles, kt0 + split_tiles);
    int pid = (int)blockIdx.x - split * total;
    {
        const int per = (total + 7) / 8, tall = total % 8 == 0 ? 8 : total % 8, xcd = pid % 8, local = pid / 8;
        pid = xcd < tall ? xcd * per + local : tall * per + (xcd - tall) * (per - 1) + local;
    }
    const int band = pid / (8 * tiles_m), in_band = pid % (8 * tiles_m), band_w = min(8, tiles_n - band * 8);
    const int n0 = (band * 8 + in_band % band_w) * C::BN, m0 = in_band / band_w * C::BM;

    // ---- fills.  LDS rows of X are 128 bytes, of W 64; slot s of a row holds granule s ^ turn(row), so that the 16 rows that a quarter of a wave reads at once
    // lie in 16 different groups of banks.  Rows past M or N fail the descriptor's check and are zero; tiles past the last have empty descriptors.
    const int64_t x_slab = (int64_t)M * KT, w_slab = (int64_t)N * SEG;
    const uint8_t *const x0 = x + (int64_t)m0 * KT, *const w0 = w + (int64_t)n0 * SEG;
    const int x_bytes = min(C::BM, M - m0) * KT, w_bytes = min(C::BN, N - n0) * SEG, s_bytes = min(C::BN, N - n0) * 4;
    const int x_even = wave * C::X_LOADS * 1024 + (lane >> 3) * KT, w_voff = wave * C::W_LOADS * 1024 + (lane >> 2) * SEG + (((lane & 3) ^ ((lane >> 4) & 3)) << 4);
    // the fills come in order, so that an addition makes the next addresses
    const uint8_t *x_next = x0 + (kt0 + kg) * x_slab, *w_next = w0 + (kt0 + kg) * w_slab;
    int kt_next = kt0 + kg;
    auto next_fill = [&](int stage, Fill &f) {
        f.live = kt_next < kt1;
        f.x = __builtin_amdgcn_make_buffer_rsrc((void *)x_next, 0, f.live ? x_bytes : 0, RSRC_FLAGS);
        f.w = __builtin_amdgcn_make_buffer_rsrc((void *)w_next, 0, f.live ? w_bytes : 0, RSRC_FLAGS);
        uint32_t first, rest;
        divide((uint32_t)kt_next, tiles_per_group, reciprocal_of_it, first, rest);
        f.base = ring + stage * C::STAGE_BYTES, f.first = (int)first * C::GT;
        x_next += C::KS * x_slab, w_next += C::KS * w_slab, kt_next += C::KS;
    };
    // load j of a fill
    auto fill = [&](const Fill &f, int j) {
        if (j < C::W_LOADS) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(f.w, LDS_PTR(f.base + C::X_BYTES + (wave * C::W_LOADS + j) * 1024), 16, w_voff + j * 1024, 0, 0, 0);
        } else if (j < C::W_LOADS + C::X_LOADS) {
            const int i = j - C::W_LOADS, chunk = wave * C::X_LOADS + i, turn = ((chunk & 1) * 4 + (lane >> 4)) & 7;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(f.x, LDS_PTR(f.base + chunk * 1024), 16, x_even + i * 1024 + (((lane & 7) ^ turn) << 4), 0, 0, 0);
        } else {
            const int i = j - C::W_LOADS - C::X_LOADS, piece = (wave * C::S_LOADS + i) % C::S_PIECES, part = piece % (C::BN / 64);
            const int group = min(f.first + piece / (C::BN / 64), groups - 1);      // a last tile may hold fewer groups: its weights there are zero
            const __amdgpu_buffer_rsrc_t sr = __builtin_amdgcn_make_buffer_rsrc((void *)(scales + (int64_t)group * N + n0), 0, f.live ? s_bytes : 0, RSRC_FLAGS);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(sr, LDS_PTR(f.base + C::X_BYTES + C::W_BYTES + piece * 256), 4, (part * 64 + lane) * 4, 0, 0, 0);
        }
    };

    float sum[C::TN][C::TM][16];
#pragma unroll
    for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
        for (int tm = 0; tm < C::TM; ++tm)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[tn][tm][r] = 0.0f;

    // ---- A K tile is UNITS units: the MFMAs of one group of one sub-tile.  While those of a unit run, the sums of the unit before are converted and added
    // (VALU instructions behind each MFMA, pinned there), the tokens' operands of the next sub-tile are read, into the registers of those that the unit is the last to use or,
    // where there is room, into others and a unit earlier, and loads of a later K tile are issued.
    constexpr int MFMAS = 4 / C::GT, UNITS = C::TN * C::TM * C::GT, LAST = UNITS - 1, FIRST = UNITS > 2 ? 1 : 0, PER_UNIT = (C::LOADS + LAST - FIRST - 1) / (LAST - FIRST);
    static_assert(UNITS % 2 == 0, "units take two sets of accumulators in turn");
    v16i none = {};
    if (C::PRESET) {
#pragma unroll
        for (int r = 0; r < 16; ++r) none[r] = 0x4b400000;
        asm volatile("" : "+v"(none));      // kept in registers: as constants they would be moved there for every unit
    }
    v16i acc[2] = {none, none};
    v4i xo[C::SETS][4], wo[C::TN][4], raw[C::TN][2];
    float sc[C::TN][C::GT], sc_last = 0.0f;
    const int steps = (kt1 - kt0 + C::KS - 1) / C::KS;      // the same for all sets: they share the barriers
    // the tokens' scales, first of all loads; waves without a piece of their own repeat another's
    {
        const __amdgpu_buffer_rsrc_t tr = __builtin_amdgcn_make_buffer_rsrc((void *)(token_scale + m0), 0, min(C::BM, M - m0) * 4, RSRC_FLAGS);
        const int piece = wave_all % C::TOKEN_PIECES;
        if (C::loads_token(piece, lane)) __builtin_amdgcn_raw_ptr_buffer_load_lds(tr, LDS_PTR(lds + C::SCALES_AT + piece * 256), 4, (piece * 64 + lane) * 4, 0, 0, 0);
    }
#pragma unroll
    for (int s = 0; s < C::STAGES - 1; ++s) {
        Fill f;
        next_fill(s, f);
#pragma unroll
        for (int j = 0; j < C::LOADS; ++j) fill(f, j);
    }
    const int x_turn = (i32 >> 1) & 7, w_turn = (i32 >> 2) & 3;
    const int x_at = (wave_m * C::TM * 32 + i32) * KT, w_at = C::X_BYTES + (wave_n * C::TN * 32 + i32) * SEG, s_at = C::X_BYTES + C::W_BYTES + (wave_n * C::TN * 32 + i32) * 4;
    // operand m of a K tile covers k = 64 (m / 2) + 32 h + 16 (m % 2) ..., or 32 m + 16 h ... where a group has 32 values
    auto read_x = [&](const uint8_t *base, int tm, int m) {
        const int granule = C::GT == 4 ? 2 * m + h : 4 * (m / 2) + 2 * h + m % 2;
        xo[tm % C::SETS][m] = *reinterpret_cast<const v4i *>(base + x_at + tm * 32 * KT + ((granule ^ x_turn) << 4));
    };
    auto read_w = [&](const uint8_t *base) {
#pragma unroll
        for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                const uint8_t *const row = base + w_at + tn * 32 * SEG;
                if constexpr (C::GT == 4) {
                    const v2i p = *reinterpret_cast<const v2i *>(row + (((2 * kk) ^ w_turn) << 4) + 8 * h), q = *reinterpret_cast<const v2i *>(row + (((2 * kk + 1) ^ w_turn) << 4) + 8 * h);
                    raw[tn][kk] = v4i{p.x, p.y, q.x, q.y};
                } else {
                    raw[tn][kk] = *reinterpret_cast<const v4i *>(row + (((2 * kk + h) ^ w_turn) << 4));
                }
            }
    };
    auto read_scales = [&](const uint8_t *base) {
#pragma unroll
        for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
            for (int g = 0; g < C::GT; ++g) sc[tn][g] = *reinterpret_cast<const float *>(base + s_at + (g * C::BN + tn * 32) * 4);
    };
    auto widen = [&](int tn) {
#pragma unroll
        for (int m = 0; m < 4; ++m) wo[tn][m] = widen2(raw[tn][m / 2][m % 2 * 2], raw[tn][m / 2][m % 2 * 2 + 1]);
    };
    auto convert = [&](const v16i &a, float s, float (&f)[16]) {
#pragma unroll
        for (int r = 0; r < 16; ++r) f[r] = __builtin_fmaf(C::PRESET ? __uint_as_float((uint32_t)a[r]) - 12582912.0f : (float)a[r], s, f[r]);
    };
    int stage = 0;
    for (int step = 0; step < steps; ++step) {
        const uint8_t *const base = ring + stage * C::STAGE_BYTES;
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(C::LOADS * (C::STAGES - 2)));      // this wave's loads of this K tile are in
        __builtin_amdgcn_s_waitcnt(WAIT_LGKM0);                                    // and its reads of the one before
        if (C::WAVES > 1) __builtin_amdgcn_s_barrier();                            // everybody's are
        __builtin_amdgcn_sched_barrier(0);
        read_w(base);
#pragma unroll
        for (int m = 0; m < 4; ++m) read_x(base, 0, m);
        read_scales(base);
        widen(0);
        Fill next;
        next_fill(stage == 0 ? C::STAGES - 1 : stage - 1, next);
        in_order(std::make_integer_sequence<int, UNITS>(), [&](auto unit) {
            constexpr int u = decltype(unit)::value, tm = u / (C::TN * C::GT), tn = u / C::GT % C::TN, g = u % C::GT, p = (u + LAST) % UNITS;
            constexpr bool reads = tn == (C::SETS == 1 ? C::TN - 1 : 0) && tm + 1 < C::TM, widening = tm == 0 && g == 0 && tn + 1 < C::TN;
            constexpr int at = (u - FIRST) * PER_UNIT, loads = u < FIRST || at >= C::LOADS ? 0 : C::LOADS - at < PER_UNIT ? C::LOADS - at : PER_UNIT;
            constexpr int valu = (32 + (widening ? 24 : 0) + MFMAS - 1) / MFMAS;
            v16i a = none;
#pragma unroll
            for (int m = 0; m < MFMAS; ++m) a = __builtin_amdgcn_mfma_i32_32x32x32_i8(xo[tm % C::SETS][g * MFMAS + m], wo[tn][g * MFMAS + m], a, 0, 0, 0);
            convert(acc[p % 2], u == 0 ? sc_last : sc[p / C::GT % C::TN][p % C::GT], sum[p / C::GT % C::TN][p / (C::TN * C::GT)]);
            acc[u % 2] = a;
            if constexpr (widening) widen(tn + 1);
            if constexpr (reads) {
#pragma unroll
                for (int m = 0; m < MFMAS; ++m) read_x(base, tm + 1, g * MFMAS + m);
            }
#pragma unroll
            for (int j = 0; j < loads; ++j) fill(next, at + j);
#pragma unroll
            for (int m = 0; m < MFMAS; ++m) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (reads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                if (loads > 0 && m == 0) __builtin_amdgcn_sched_group_barrier(0x010, loads > 0 ? loads : 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, valu, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        sc_last = sc[C::TN - 1][C::GT - 1];
        stage = stage + 1 == C::STAGES ? 0 : stage + 1;
    }
    convert(acc[LAST % 2], sc_last, sum[C::TN - 1][C::TM - 1]);
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));      // loads past the last tile, which write LDS

    // ---- epilogue, 32 tokens of each wave at a time: the sums go to LDS as [set][token][channel] and come back four channels of a token to a thread, whose sets it
    // adds in order.  Register r of lane (i, h) is token 8 (r / 4) + 4 h + r % 4, channel i of its sub-tile.
    float *const out = reinterpret_cast<float *>(lds);
    const float *const token_scales = reinterpret_cast<const float *>(lds + C::SCALES_AT);
    constexpr int PIECES = C::OUT_ROWS * C::BN / 4 / C::THREADS, SET = C::OUT_ROWS * C::BN;
    const int n = n0 + (tid * 4) % C::BN;
    __syncthreads();
#pragma unroll
    for (int tm = 0; tm < C::TM; ++tm) {
        float *const pass = out + tm % C::PASSES * (C::KS * SET);
        if (C::PASSES == 1 && tm > 0) __syncthreads();
#pragma unroll
        for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                pass[kg * SET + (wave_m * 32 + 8 * (r / 4) + 4 * h + r % 4) * C::BN + (wave_n * C::TN + tn) * 32 + i32] = sum[tn][tm][r];
        __syncthreads();
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int at = (p * C::THREADS + tid) * 4, row = at / C::BN, of_tile = (row / 32 * C::TM + tm) * 32 + row % 32, t = m0 + of_tile;
            if (t >= M || n >= N) continue;
            v4f v = *reinterpret_cast<const v4f *>(pass + at);
#pragma unroll
            for (int k = 1; k < C::KS; ++k) v += *reinterpret_cast<const v4f *>(pass + k * SET + at);
            if (y_type == PARTIAL) {
                const int64_t stride = (N + 3) / 4 * 4;
                *reinterpret_cast<v4f *>(static_cast<float *>(y) + ((int64_t)split * M + t) * stride + n) = v;
                continue;
            }
            store_four(v, token_scales[of_tile], t, n, N, y, y_type);
        }
    }
}

// The sums of all splits of a problem, in order; a thread takes four channels of a token.
__global__ __launch_bounds__(256) void grouped_join_kernel(const float *__restrict__ parts, int splits, int M, int N, const float *__restrict__ token_scale, void *__restrict__ y,
                                                           int y_type)
{
    const int pieces = (N + 3) / 4;
    const int64_t total = (int64_t)M * pieces, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const int t = (int)(i / pieces), n = (int)(i % pieces) * 4;
    v4f v = *reinterpret_cast<const v4f *>(parts + i * 4);
    for (int s = 1; s < splits; ++s) v += *reinterpret_cast<const v4f *>(parts + (s * total + i) * 4);
    store_four(v, token_scale[t], t, n, N, y, y_type);
}

// ---- which kernel
//
// What a tile shape's launch takes, in us, fitted on 6032 problems of random sizes (17 to 6000 tokens, 256 to 60000 channels, K up to 16384, weights not in any cache; about 2700 of them in
// groups of 128, 1500 in groups of 64, 1800 in groups of 32), each run with every shape on an MI355X: `start`, and for every CU, `fit` workgroups at a time, `fixed` and `step` a K tile of
// a set, which depend on how many run there together.  Against the best of these ten and of four few-token kernels the choice takes, from 65 tokens on, 0.3 to 0.8 % longer on average
// and 2 to 6 % at the 95th percentile, and up to 64 tokens 1.3 to 2.0 and 8 to 11 %.  Without 256 x 128 and 256 x 96 the best would take 0.5 to 2 % longer, where a call's tiles then make another round
// of the CUs 10 to 20 (96 x 57344 x 8192 93 us, on 256 x 96 76; 700 x 8192 x 8192 76 and 63).
struct TileCost {
    int bn, bm, sets, fit;
    float start, fixed[3], step[3];
};
constexpr int TILES = 10;
constexpr TileCost COSTS[3][TILES] = {      // groups of 128 and more, of 64, of 32 (zeros: no such kernel)
    {
        {256, 256, 1, 1, 0.00f, {9.07f}, {1.62f}},
        {256, 192, 1, 1, 0.42f, {7.14f}, {1.33f}},
        {256, 128, 2, 1, 0.86f, {6.11f}, {1.72f}},
        {256, 96, 2, 1, 1.25f, {4.46f}, {1.53f}},
        {256, 64, 2, 1, 1.35f, {3.74f}, {1.07f}},
        {128, 64, 1, 3, 2.90f, {0.98f, 1.96f, 2.77f}, {0.51f, 0.70f, 0.94f}},
        {128, 64, 2, 1, 1.38f, {2.72f}, {0.61f}},
        {128, 32, 2, 2, 2.48f, {1.16f, 2.16f}, {0.56f, 0.74f}},
        {64, 64, 4, 1, 1.44f, {2.93f}, {0.72f}},
        {64, 32, 8, 1, 1.54f, {2.03f}, {0.78f}},
    },
    {
        {256, 256, 1, 1, 0.00f, {9.19f}, {2.25f}},
        {256, 192, 1, 1, 0.65f, {6.99f}, {1.73f}},
        {256, 128, 2, 1, 1.27f, {5.94f}, {2.33f}},
        {256, 96, 2, 1, 1.40f, {4.69f}, {1.87f}},
        {256, 64, 2, 1, 1.40f, {3.81f}, {1.34f}},
        {128, 64, 1, 3, 2.89f, {1.01f, 2.07f, 2.67f}, {0.58f, 0.77f, 1.11f}},
        {128, 64, 2, 1, 1.43f, {2.70f}, {0.77f}},
        {128, 32, 2, 2, 2.64f, {1.02f, 2.21f}, {0.65f, 0.87f}},
        {64, 64, 4, 1, 1.52f, {2.84f}, {0.92f}},
        {64, 32, 8, 1, 1.61f, {1.95f}, {0.91f}},
    },
    {
        {256, 256, 1, 1, 0.00f, {0.00f}, {0.00f}},
        {256, 192, 1, 1, 0.33f, {7.41f}, {2.56f}},
        {256, 128, 2, 1, 0.00f, {0.00f}, {0.00f}},
        {256, 96, 2, 1, 1.05f, {5.05f}, {2.65f}},
        {256, 64, 2, 1, 0.00f, {0.00f}, {0.00f}},
        {128, 64, 1, 2, 2.53f, {1.32f, 2.59f}, {0.83f, 1.07f}},
        {128, 64, 2, 1, 1.27f, {2.82f}, {1.05f}},
        {128, 32, 2, 1, 1.67f, {2.24f}, {0.87f}},
        {64, 64, 4, 1, 1.40f, {2.92f}, {1.40f}},
        {64, 32, 8, 1, 1.56f, {1.99f}, {1.24f}},
    },
};
constexpr float JOIN_START = 3.0f, JOIN_BYTE = 0.4e-6f;      // us: the second launch of a split K, and a byte of its ranges' sums, written and read
template <int GT> using Tile0 = Tile<4, 2, 2, 4, 3, 1, GT>;
template <int GT> using Tile1 = Tile<4, 2, 2, 3, 3, 1, GT>;
template <int GT> using Tile2 = Tile<4, 1, 2, 4, 2, 2, GT>;
template <int GT> using Tile3 = Tile<4, 1, 2, 3, 2, 2, GT>;
template <int GT> using Tile4 = Tile<4, 1, 2, 2, 3, 2, GT>;
template <int GT> using Tile5 = Tile<2, 2, 2, 1, 3, 1, GT>;
template <int GT> using Tile6 = Tile<4, 1, 1, 2, 3, 2, GT>;
template <int GT> using Tile7 = Tile<2, 1, 2, 1, 3, 2, GT>;
template <int GT> using Tile8 = Tile<1, 1, 2, 2, 3, 4, GT>;
template <int GT> using Tile9 = Tile<1, 1, 2, 1, 2, 8, GT>;
// groups of 32: 256 x 256 and 256 x 128 would spill (3 and 7 registers), 256 x 64 has no room for its scales in LDS (172288 bytes)
constexpr bool tile_serves(int i, int gt) { return gt < 4 || (i != 0 && i != 2 && i != 4); }

// Workgroups of a tile kernel that a CU's LDS holds, given out in pieces of 1280 bytes; the table may not count on more.
template <class C>
constexpr int lds_room()
{
    return 160 * 1024 / ((C::LDS_BYTES + 1279) / 1280 * 1280);
}
template <int GT>
constexpr bool fit_in_lds()
{
    const TileCost(&costs)[TILES] = COSTS[GT >> 1];
    bool fit = costs[1].fit <= lds_room<Tile1<GT>>() && costs[3].fit <= lds_room<Tile3<GT>>() && costs[5].fit <= lds_room<Tile5<GT>>() && costs[6].fit <= lds_room<Tile6<GT>>() &&
               costs[7].fit <= lds_room<Tile7<GT>>() && costs[8].fit <= lds_room<Tile8<GT>>() && costs[9].fit <= lds_room<Tile9<GT>>();
    if constexpr (tile_serves(0, GT)) fit = fit && costs[0].fit <= lds_room<Tile0<GT>>();
    if constexpr (tile_serves(2, GT)) fit = fit && costs[2].fit <= lds_room<Tile2<GT>>();
    if constexpr (tile_serves(4, GT)) fit = fit && costs[4].fit <= lds_room<Tile4<GT>>();
    return fit;
}
static_assert(fit_in_lds<1>() && fit_in_lds<2>() && fit_in_lds<4>(), "more workgroups than LDS holds");

static int64_t tiles_of(const TileCost &c, int64_t M, int64_t N) { return ((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn); }

static float tile_estimate(const TileCost &c, int64_t workgroups, int64_t kt, int64_t cus)
{
    const int64_t each = (workgroups + cus - 1) / cus, full = each / c.fit, rest = each % c.fit;      // workgroups of a CU
    const float steps = (float)((kt + c.sets - 1) / c.sets);
    return c.start + (float)full * (c.fixed[c.fit - 1] + steps * c.step[c.fit - 1]) + (rest ? c.fixed[rest - 1] + steps * c.step[rest - 1] : 0.0f);
}

// The few-token kernels the same way: a start, and for every K tile of a wave a latency and what each workgroup of a CU adds.
struct FewCost {
    int waves, channels;
    float start, latency, each;
};
constexpr FewCost FEW_COSTS[3][3] = {{{16, 16, 1.82f, 0.37f, 0.79f}, {16, 32, 1.52f, 0.57f, 1.10f}, {8, 32, 2.27f, 0.14f, 0.62f}},
                                     {{16, 16, 1.74f, 0.34f, 0.90f}, {16, 32, 1.62f, 0.59f, 1.08f}, {8, 32, 2.35f, 0.12f, 0.67f}},
                                     {{16, 16, 0.85f, 1.27f, 1.07f}, {16, 32, 0.90f, 1.33f, 1.38f}, {8, 32, 2.12f, 0.38f, 0.87f}}};

static float few_estimate(const FewCost &c, int64_t M, int64_t N, int64_t kt, int64_t cus)
{
    const int64_t steps = (kt + c.waves - 1) / c.waves, each = ((N + c.channels - 1) / c.channels * ((M + 15) / 16) + cus - 1) / cus;
    return c.start + (float)steps * (c.latency + (float)each * c.each);
}

static int64_t partial_bytes(int64_t M, int64_t N) { return M * ((N + 3) / 4 * 16); }      // of the sums of a range of K

// What a call takes: 0 .. 9 a tile, 10 + i the few-token kernel FEW_COSTS[..][i], 13 the one of eight waves and 16 channels; into how many ranges K is split between workgroups.
struct Choice {
    int kernel, splits;
};

// Up to 16 tokens, on 10188 matrices of up to 130000 channels with groups of 128 and 64, by two lines:
// short K wants eight waves; as many workgroups as CUs or a few times as many want sixteen waves, with 32 channels from 16 * CUs channels on; more workgroups want eight
// again while K is not long.  us, 16 waves of 16 channels / 16 of 32 / 8 of 16 / 8 of 32: 4096 x 14336 7.8 / 8.9 / 10.6 / 14, 6144 x 4096 5.1 / 4.6 / 4.9 / 5.2, 28672 x 4096 - / 13.2 / 13.5 / 12.3.
// From 13 tokens on such a kernel reads as many bytes of tokens as of weights, and a long K against many channels wants tiles (sixteen waves of
// 32 channels / tile: 15 x 9600 x 13952 24.0 / 20.0, 16 x 30656 x 14080 55.3 / 46.3).  The choice takes 0.3 to 1.5 % longer than the best kernel on average, with 13 to 16 tokens and more than 64M weights 2 to 4 %.
static Choice grouped_choice(int64_t M, int64_t N, int64_t K, int gt, int64_t scratch)
{
    const int64_t kt = k_tiles(K), cus = device_cus_or_default();
    if (M <= 16) {
        if (M > 12 && kt >= 32 && N > 32 * cus && N <= 64 * cus) return {9, 1};
        if (M > 12 && kt >= 48 && N > 96 * cus) return {gt == 4 ? 9 : 7, 1};
        if (kt < 9) return {N <= 48 * cus ? 13 : 12, 1};
        return {N <= 16 * cus ? 10 : N > 64 * cus && kt < 33 ? 12 : 11, 1};
    }
    // no kernel takes less than its bytes do at 4.8 TB/s; among those that come to it the larger tile reads less (32 x 28672 x 4096, 128 x 32 14.4 us, 64 x 32 17.0)
    const float bytes = (float)N * (float)kt * (float)(SEG + 4 * gt) + (float)M * (float)kt * (float)KT + 2.0f * (float)M * (float)N, memory = bytes / 4.8e6f;
    const TileCost *const costs = COSTS[gt >> 1];
    Choice best = {-1, 1};
    float least = 0.0f;
    auto offer = [&](int i, int splits, float us) {
        us = us > memory ? us : memory;
        if (best.kernel < 0 || us < least) best = {i, splits}, least = us;
    };
    for (int i = 0; i < TILES; ++i)
        if (tile_serves(i, gt)) offer(i, 1, tile_estimate(costs[i], tiles_of(costs[i], M, N), kt, cus));
    if (M <= 64)
        for (int i = 0; i < 3; ++i) offer(TILES + i, 1, few_estimate(FEW_COSTS[gt >> 1][i], M, N, kt, cus));
    // Few tiles and a long K: its ranges go to workgroups of their own, and a second launch adds their sums.
    const int64_t range = partial_bytes(M, N);
    for (int i = 0; i < TILES; ++i) {
        const int64_t tiles = tiles_of(costs[i], M, N);
        for (int splits = 2; splits <= 8 && tile_serves(i, gt) && tiles * splits <= 2 * cus && kt / splits >= 8 && splits * range <= scratch; ++splits)
            offer(i, splits, tile_estimate(costs[i], tiles * splits, (kt + splits - 1) / splits, cus) + JOIN_START + (float)(splits * range) * JOIN_BYTE);
    }
    return best;
}

template <class C>
static hipError_t set_tile_attribute()
{
    return hipFuncSetAttribute((const void *)grouped_tile_kernel<C>, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES);
}
template <int GT>
static hipError_t set_tile_attributes()
{
    hipError_t e = hipSuccess;
    if constexpr (tile_serves(0, GT)) e = set_tile_attribute<Tile0<GT>>();
    if (e == hipSuccess) e = set_tile_attribute<Tile1<GT>>();
    if constexpr (tile_serves(2, GT)) e = e == hipSuccess ? set_tile_attribute<Tile2<GT>>() : e;
    if (e == hipSuccess) e = set_tile_attribute<Tile3<GT>>();
    if constexpr (tile_serves(4, GT)) e = e == hipSuccess ? set_tile_attribute<Tile4<GT>>() : e;
    if (e == hipSuccess) e = set_tile_attribute<Tile5<GT>>();
    if (e == hipSuccess) e = set_tile_attribute<Tile6<GT>>();
    if (e == hipSuccess) e = set_tile_attribute<Tile7<GT>>();
    if (e == hipSuccess) e = set_tile_attribute<Tile8<GT>>();
    return e == hipSuccess ? set_tile_attribute<Tile9<GT>>() : e;
}
hipError_t grouped_device_init()
{
    hipError_t e = set_tile_attributes<1>();
    if (e == hipSuccess) e = set_tile_attributes<2>();
    return e == hipSuccess ? set_tile_attributes<4>() : e;
}

struct GroupedCall {
    const uint8_t *x;
    const float *token_scale;
    const uint8_t *w;
    int M, N, ktiles, groups;
    uint32_t per;      // K tiles of a group
    const float *scales;
    void *y;
    int y_type;
    hipStream_t stream;
    int splits;
    float *parts;
};

template <class C>
static hipError_t launch_tile(const GroupedCall &c)
{
    const int64_t tiles_m = (c.M + C::BM - 1) / C::BM, tiles_n = (c.N + C::BN - 1) / C::BN;
    if (tiles_m * tiles_n * c.splits > (int64_t)0xffffffff / C::THREADS) return hipErrorInvalidConfiguration;
    const DeviceInfo *info;
    const hipError_t e = device_info(&info);      // the tiles' LDS is an attribute of the kernels, set once per device
    if (e != hipSuccess) return e;
    const bool split = c.splits > 1;
    grouped_tile_kernel<C><<<dim3((unsigned)(tiles_m * tiles_n * c.splits)), dim3(C::THREADS), C::LDS_BYTES, c.stream>>>(
        c.x, c.w, c.scales, c.M, c.N, c.ktiles, (int)tiles_m, (int)tiles_n, c.per, reciprocal(c.per), c.groups, c.token_scale, split ? c.parts : c.y,
        split ? PARTIAL : c.y_type, (c.ktiles + c.splits - 1) / c.splits);
    if (!split) return hipGetLastError();
    const hipError_t launched = hipGetLastError();
    if (launched != hipSuccess) return launched;
    const int64_t pieces = (int64_t)c.M * ((c.N + 3) / 4);
    grouped_join_kernel<<<dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, c.stream>>>(c.parts, c.splits, c.M, c.N, c.token_scale, c.y, c.y_type);
    return hipGetLastError();
}

template <int WAVES, int RT, int GT>
static hipError_t launch_few(const GroupedCall &c)
{
    grouped_few_kernel<WAVES, RT, GT><<<dim3((unsigned)((c.N + 16 * RT - 1) / (16 * RT)), (unsigned)((c.M + 15) / 16)), dim3(64 * WAVES), 0, c.stream>>>(
        c.x, c.w, c.scales, c.M, c.N, c.ktiles, c.groups, c.per, reciprocal(c.per), c.token_scale, c.y, c.y_type);
    return hipGetLastError();
}

template <int GT>
static hipError_t launch_choice(int choice, const GroupedCall &c)
{
    switch (choice) {
    case 0:
        if constexpr (tile_serves(0, GT)) return launch_tile<Tile0<GT>>(c);
        break;
    case 1: return launch_tile<Tile1<GT>>(c);
    case 2:
        if constexpr (tile_serves(2, GT)) return launch_tile<Tile2<GT>>(c);
        break;
    case 3: return launch_tile<Tile3<GT>>(c);
    case 4:
        if constexpr (tile_serves(4, GT)) return launch_tile<Tile4<GT>>(c);
        break;
    case 5: return launch_tile<Tile5<GT>>(c);
    case 6: return launch_tile<Tile6<GT>>(c);
    case 7: return launch_tile<Tile7<GT>>(c);
    case 8: return launch_tile<Tile8<GT>>(c);
    case 9: return launch_tile<Tile9<GT>>(c);
    case 10: return launch_few<16, 1, GT>(c);
    case 11: return launch_few<16, 2, GT>(c);
    case 12: return launch_few<8, 2, GT>(c);
    case 13: return launch_few<8, 1, GT>(c);
    }
    return hipErrorInvalidValue;
}

// 0: chosen per problem; 1 + i forces kernel i, in as many ranges of K as splits says where there is scratch (testing and tuning)
static std::atomic<int> g_forced_grouped{0};
bool set_grouped_kernel(int kernel, int splits)
{
    if (kernel < 0 || kernel > TILES + 4 || splits < 1 || splits > 8) return false;
    g_forced_grouped.store(kernel + 16 * splits, std::memory_order_relaxed);
    return true;
}

static Choice chosen(int64_t M, int64_t N, int64_t K, int64_t group, int64_t scratch)
{
    const int code = g_forced_grouped.load(std::memory_order_relaxed), forced = code % 16, splits = code / 16;
    if (!forced) return grouped_choice(M, N, K, group == 32 ? 4 : group == 64 ? 2 : 1, scratch);
    const bool room = forced <= TILES && splits <= k_tiles(K) && splits * partial_bytes(M, N) <= scratch;
    return {forced - 1, room ? splits : 1};
}

constexpr int64_t MOST_SCRATCH = (int64_t)64 << 20;
int64_t grouped_scratch_bytes(int64_t M, int64_t N, int64_t K, int64_t group)
{
    const Choice c = chosen(M, N, K, group, MOST_SCRATCH);
    return c.splits > 1 ? c.splits * partial_bytes(M, N) : 0;
}
int grouped_kernel(int64_t M, int64_t N, int64_t K, int64_t group) { return chosen(M, N, K, group, 0).kernel; }

hipError_t launch_grouped_linear(const uint8_t *x, const float *token_scale, const uint8_t *w, int64_t M, int64_t N, int64_t K, int64_t group, const float *scales,
                                 void *y, int y_type, void *scratch, int64_t scratch_bytes, hipStream_t s)
{
    const int64_t kt = k_tiles(K), per = group > KT ? (group / KT < kt ? group / KT : kt) : 1;
    Choice choice = chosen(M, N, K, group, scratch ? MOST_SCRATCH : 0);
    if (choice.splits > 1 && choice.splits * partial_bytes(M, N) > scratch_bytes) choice = chosen(M, N, K, group, 0);      // too little counts as none, so that results depend on one thing less
    const GroupedCall c = {x, token_scale, w, (int)M, (int)N, (int)kt, (int)((K - 1) / group + 1), (uint32_t)per, scales, y, y_type, s, choice.splits, (float *)scratch};
    return group == 32 ? launch_choice<4>(choice.kernel, c) : group == 64 ? launch_choice<2>(choice.kernel, c) : launch_choice<1>(choice.kernel, c);
}

}  // namespace fptq
