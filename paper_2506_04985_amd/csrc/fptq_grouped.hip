// Linear layer of 8-bit activations and packed 4-bit weights with a scale for each group of K values:
//     y[t, n] = s_t * sum_g s[g, n] * (sum over k in g of code[t, k] * w[n, k])
// The inner sum is an integer and exact; those of the groups are added in fp32.
//
// Nibbles are widened to bytes that hold 16 * value as in the other linears, (p << 4) & 0xF0F0F0F0 and p & 0xF0F0F0F0, and the codes of eight k lie
// in that order, so they are operands as they are.  Of 128 k or fewer, 16 * sum stays below 2^21 in magnitude, which fp32 holds exactly; the 1/16 goes into the
// token's scale, exactly as well.  Groups of several K tiles take their scale once a tile.
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

// A workgroup owns 16 RT channels, its waves split K (wave w takes K tiles w, w + WAVES, ...), MT groups of 16 tokens.  Tokens are the rows of the MFMA's
// result and channels its columns, so that a lane has one channel, and one scale of it a group.
template <int WAVES, int U, int MT, int RT, int GT>
__global__ __launch_bounds__(64 * WAVES) void grouped_few_kernel(const uint8_t *__restrict__ x, const uint8_t *__restrict__ w, const float *__restrict__ scales, int M,
                                                                 int N, int ktiles, int groups, uint32_t tiles_per_group, uint32_t reciprocal_of_it,
                                                                 const float *__restrict__ token_scale, void *__restrict__ y, int y_type)
{
    __shared__ float red[WAVES][RT * MT * 256];
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = blockIdx.x * (16 * RT), m0 = blockIdx.y * (16 * MT);
    const int64_t w_slab = (int64_t)N * SEG, x_slab = (int64_t)M * KT;
    const uint8_t *wp[RT], *xp[MT];
    const float *sp[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int n = min(n0 + rt * 16 + c, N - 1);
        wp[rt] = w + (int64_t)n * SEG + q * 16;
        sp[rt] = scales + n;
    }
    // a token's 16 or 8 codes for each MFMA, as by_group leaves the weights
    constexpr int STEPS = GT == 4 ? 4 : 2;
    const int x_first = GT == 1 ? q * 32 : GT == 2 ? (q & 1) * 32 + (q >> 1) * 16 : q * 8;
    constexpr int x_step = GT == 1 ? 16 : GT == 2 ? 64 : 32;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) xp[mt] = x + (int64_t)min(m0 + mt * 16 + c, M - 1) * KT + x_first;

    v4f sum[RT][MT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sum[rt][mt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const int T = wave < ktiles ? (ktiles - wave + WAVES - 1) / WAVES : 0;
    for (int base = 0; base < T; base += U) {
        v4i wv[RT][U];
        float sv[RT][U][GT];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (base + u < T) {
                const int64_t kt = wave + (base + u) * WAVES;
                uint32_t first, rest;
                divide((uint32_t)kt, tiles_per_group, reciprocal_of_it, first, rest);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    wv[rt][u] = __builtin_nontemporal_load(reinterpret_cast<const v4i *>(wp[rt] + kt * w_slab));
#pragma unroll
                    for (int g = 0; g < GT; ++g)      // a last tile may hold fewer groups: its weights there are zero
                        sv[rt][u][g] = sp[rt][(int64_t)min((int)first * GT + g, groups - 1) * N];
                }
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (base + u < T) {
                const int64_t kt = wave + (base + u) * WAVES;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    v4i xv[STEPS];
#pragma unroll
                    for (int j = 0; j < STEPS; ++j) {
                        if (GT == 4) {
                            const v2i v = *reinterpret_cast<const v2i *>(xp[mt] + kt * x_slab + j * x_step);
                            xv[j] = v4i{v.x, v.y, 0, 0};
                        } else {
                            xv[j] = *reinterpret_cast<const v4i *>(xp[mt] + kt * x_slab + j * x_step);
                        }
                    }
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        v4i wd = wv[rt][u];
                        by_group<GT>(wd);
                        v4i acc = {0, 0, 0, 0};
#pragma unroll
                        for (int j = 0; j < STEPS; ++j) {
                            if constexpr (GT == 4) {
                                const v2i b = widen1(wd[j]);
                                acc = __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, v2i{xv[j].x, xv[j].y}), __builtin_bit_cast(long, b), v4i{0, 0, 0, 0}, 0, 0, 0);
                            } else {
                                acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(xv[j], widen2(wd[2 * j], wd[2 * j + 1]), GT == 2 ? v4i{0, 0, 0, 0} : acc, 0, 0, 0);
                            }
                            if (GT != 1 || j == 1) {
                                const float s = sv[rt][u][GT == 1 ? 0 : j];
#pragma unroll
                                for (int r = 0; r < 4; ++r) sum[rt][mt][r] = __builtin_fmaf((float)acc[r], s, sum[rt][mt][r]);
                            }
                        }
                    }
                }
            }
    }

    // lane l, register r holds token 4 (l / 16) + r, channel l % 16
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r) red[wave][(mt * 16 + 4 * q + r) * (16 * RT) + rt * 16 + c] = sum[rt][mt][r];
    __syncthreads();
    for (int o = tid; o < RT * MT * 256; o += 64 * WAVES) {
        float v = red[0][o];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v += red[i][o];
        const int t = m0 + o / (16 * RT), n = n0 + o % (16 * RT);
        if (t < M && n < N) {
            v *= token_scale[t] * 0.0625f;
            if (y_type == FPTQ_F32)
                static_cast<float *>(y)[(int64_t)t * N + n] = v;
            else
                static_cast<uint16_t *>(y)[(int64_t)t * N + n] = bf16_rne(v);
        }
    }
}

// ---- tiles, for more tokens than a few
//
// A workgroup makes BN channels x BM tokens, each of its waves TN x TM sub-tiles of 32 x 32.  A K tile of both operands and its groups' scales go from HBM to LDS
// by loads that write LDS directly, STAGES deep, one barrier a K tile.  v_mfma_i32_32x32x32_i8 makes a group's integer sums, which go into the fp32 sums at once: with tokens
// as rows of the result and channels as columns a lane has one channel of a sub-tile, so its scale is one register, and (float)sum and a fused multiply-add are the 32
// vector instructions that 4 MFMAs (128 cycles) of a 128-value group cost.  Two waves a SIMD, so that one's conversions run under the other's MFMAs.
typedef int v16i __attribute__((ext_vector_type(16)));

template <int WAVES_N_, int WAVES_M_, int TN_, int TM_, int STAGES_, int GT_>
struct Tile {
    static constexpr int WAVES_N = WAVES_N_, WAVES_M = WAVES_M_, TN = TN_, TM = TM_, STAGES = STAGES_, GT = GT_;
    static constexpr int BN = WAVES_N * TN * 32, BM = WAVES_M * TM * 32, WAVES = WAVES_N * WAVES_M, THREADS = 64 * WAVES;
    static constexpr int X_BYTES = BM * KT, W_BYTES = BN * SEG, S_BYTES = BN * GT * 4, STAGE_BYTES = X_BYTES + W_BYTES + S_BYTES;
    static constexpr int X_LOADS = X_BYTES / (WAVES * 1024), W_LOADS = W_BYTES / (WAVES * 1024), S_PIECES = BN * GT / 64, S_LOADS = (S_PIECES + WAVES - 1) / WAVES;
    static constexpr int LOADS = X_LOADS + W_LOADS + S_LOADS, LDS_BYTES = STAGES * STAGE_BYTES;
    static_assert(X_BYTES % (WAVES * 1024) == 0 && W_BYTES % (WAVES * 1024) == 0 && BN % 64 == 0, "a K tile is shared out evenly");
    static_assert(S_PIECES % WAVES == 0 || WAVES % S_PIECES == 0, "waves without a piece of their own repeat another's");
    static_assert(LOADS * (STAGES - 1) < 64, "the count of loads in flight has six bits");
};

template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void grouped_tile_kernel(const uint8_t *__restrict__ x, const uint8_t *__restrict__ w, const float *__restrict__ scales, int M, int N,
                                                                  int ktiles, int tiles_m, int tiles_n, uint32_t tiles_per_group, uint32_t reciprocal_of_it, int groups,
                                                                  const float *__restrict__ token_scale, void *__restrict__ y, int y_type)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wave_n = wave % C::WAVES_N, wave_m = wave / C::WAVES_N, i32 = lane & 31, h = lane >> 5;

    // Workgroups go round the 8 XCDs; each gets a contiguous run of tiles, in bands of 8 along n, so that tiles that run together share operands in its L2.
    const int total = tiles_m * tiles_n;
    int pid = blockIdx.x;
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
    auto fill = [&](int kt, int stage) {
        uint8_t *const base = lds + stage * C::STAGE_BYTES;
        const bool live = kt < ktiles;
        uint32_t first, rest;
        divide((uint32_t)kt, tiles_per_group, reciprocal_of_it, first, rest);
        const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc((void *)(x0 + kt * x_slab), 0, live ? x_bytes : 0, RSRC_FLAGS);
        const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc((void *)(w0 + kt * w_slab), 0, live ? w_bytes : 0, RSRC_FLAGS);
#pragma unroll
        for (int j = 0; j < C::X_LOADS; ++j) {
            const int chunk = wave * C::X_LOADS + j, turn = ((chunk & 1) * 4 + (lane >> 4)) & 7;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, LDS_PTR(base + chunk * 1024), 16, x_even + j * 1024 + (((lane & 7) ^ turn) << 4), 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < C::W_LOADS; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, LDS_PTR(base + C::X_BYTES + (wave * C::W_LOADS + j) * 1024), 16, w_voff + j * 1024, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < C::S_LOADS; ++j) {
            const int piece = (wave * C::S_LOADS + j) % C::S_PIECES, g = piece / (C::BN / 64), part = piece % (C::BN / 64);
            const int group = (int)first * C::GT + g;
            const __amdgpu_buffer_rsrc_t sr = __builtin_amdgcn_make_buffer_rsrc((void *)(scales + (int64_t)min(group, groups - 1) * N + n0), 0, live ? s_bytes : 0, RSRC_FLAGS);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(sr, LDS_PTR(base + C::X_BYTES + C::W_BYTES + piece * 256), 4, (part * 64 + lane) * 4, 0, 0, 0);
        }
    };

    float sum[C::TN][C::TM][16];
#pragma unroll
    for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
        for (int tm = 0; tm < C::TM; ++tm)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[tn][tm][r] = 0.0f;

#pragma unroll
    for (int s = 0; s < C::STAGES - 1; ++s) fill(s, s);
    int stage = 0;
    for (int kt = 0; kt < ktiles; ++kt) {
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(C::LOADS * (C::STAGES - 2)));      // this wave's loads of tile kt are in
        __builtin_amdgcn_s_waitcnt(WAIT_LGKM0);                                    // and its reads of tile kt - 1
        __builtin_amdgcn_s_barrier();                                              // everybody's are, and everybody is done with tile kt - 1
        __builtin_amdgcn_sched_barrier(0);
        fill(kt + C::STAGES - 1, stage == 0 ? C::STAGES - 1 : stage - 1);
        const uint8_t *const base = lds + stage * C::STAGE_BYTES;
        const uint8_t *const xb = base + (wave_m * C::TM * 32 + i32) * KT;
        const uint8_t *const wb = base + C::X_BYTES + (wave_n * C::TN * 32 + i32) * SEG;
        const float *const sb = reinterpret_cast<const float *>(base + C::X_BYTES + C::W_BYTES) + wave_n * C::TN * 32 + i32;
        const int x_turn = (i32 >> 1) & 7, w_turn = (i32 >> 2) & 3;

        // operand m of a K tile covers k = 64 (m / 2) + 32 h + 16 (m % 2) ..., or 32 m + 16 h ... where a group has 32 values
        v4i wo[C::TN][4];
        float sc[C::TN][C::GT];
#pragma unroll
        for (int tn = 0; tn < C::TN; ++tn) {
            if constexpr (C::GT == 4) {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const v2i p = *reinterpret_cast<const v2i *>(wb + tn * 32 * SEG + ((m ^ w_turn) << 4) + 8 * h);
                    wo[tn][m] = widen2(p.x, p.y);
                }
            } else {
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    const v4i p = *reinterpret_cast<const v4i *>(wb + tn * 32 * SEG + (((2 * kk + h) ^ w_turn) << 4));
                    wo[tn][2 * kk] = widen2(p.x, p.y), wo[tn][2 * kk + 1] = widen2(p.z, p.w);
                }
            }
#pragma unroll
            for (int g = 0; g < C::GT; ++g) sc[tn][g] = sb[g * C::BN + tn * 32];
        }
#pragma unroll
        for (int tm = 0; tm < C::TM; ++tm) {
            v4i xo[4];
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const int granule = C::GT == 4 ? 2 * m + h : 4 * (m / 2) + 2 * h + m % 2;
                xo[m] = *reinterpret_cast<const v4i *>(xb + tm * 32 * KT + ((granule ^ x_turn) << 4));
            }
#pragma unroll
            for (int tn = 0; tn < C::TN; ++tn) {
#pragma unroll
                for (int g = 0; g < C::GT; ++g) {
                    v16i acc = {};
#pragma unroll
                    for (int m = 0; m < 4 / C::GT; ++m) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(xo[g * (4 / C::GT) + m], wo[tn][g * (4 / C::GT) + m], acc, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum[tn][tm][r] = __builtin_fmaf((float)acc[r], sc[tn][g], sum[tn][tm][r]);
                }
            }
        }
        stage = stage + 1 == C::STAGES ? 0 : stage + 1;
    }

    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));      // loads past the last tile, which write LDS

    // ---- register r of lane (i, h) is token 8 (r / 4) + 4 h + r % 4, channel i of its sub-tile.  bf16: neighbouring lanes exchange, so that each has two channels of one token.
#pragma unroll
    for (int tm = 0; tm < C::TM; ++tm) {
        const int t0 = m0 + (wave_m * C::TM + tm) * 32 + 4 * h;
        float ts[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) ts[r] = token_scale[min(t0 + 8 * (r / 4) + r % 4, M - 1)] * 0.0625f;
#pragma unroll
        for (int tn = 0; tn < C::TN; ++tn) {
            const int n = n0 + (wave_n * C::TN + tn) * 32 + i32;
            if (y_type == FPTQ_F32) {
                float *const out = static_cast<float *>(y);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int t = t0 + 8 * (r / 4) + r % 4;
                    if (t < M && n < N) out[(int64_t)t * N + n] = sum[tn][tm][r] * ts[r];
                }
            } else {
                uint16_t *const out = static_cast<uint16_t *>(y);
#pragma unroll
                for (int r = 0; r < 16; r += 2) {
                    const float a = sum[tn][tm][r] * ts[r], b = sum[tn][tm][r + 1] * ts[r + 1];
                    const bool odd = lane & 1;
                    const float theirs = __uint_as_float(other_lane<1>(__float_as_uint(odd ? a : b)));
                    const uint32_t pair = odd ? pack_bf16(theirs, b) : pack_bf16(a, theirs);
                    const int t = t0 + 8 * (r / 4) + r % 4 + (odd ? 1 : 0), c = n & ~1;
                    if (t < M) {
                        uint16_t *const to = out + (int64_t)t * N + c;
                        if (c + 1 < N)
                            __builtin_memcpy(to, &pair, 4);
                        else if (c < N)
                            *to = (uint16_t)pair;
                    }
                }
            }
        }
    }
}

template <int GT> using Large = Tile<4, 2, 2, 4, 3, GT>;      // 256 x 256
template <int GT> using Small = Tile<2, 2, 2, 2, 3, GT>;      // 128 x 128, two workgroups a CU

template <class... Cs>
static hipError_t set_tile_attributes()
{
    hipError_t e = hipSuccess;
    ((e = e == hipSuccess ? hipFuncSetAttribute((const void *)grouped_tile_kernel<Cs>, hipFuncAttributeMaxDynamicSharedMemorySize, Cs::LDS_BYTES) : e), ...);
    return e;
}
hipError_t grouped_device_init() { return set_tile_attributes<Large<1>, Large<2>, Large<4>, Small<1>, Small<2>, Small<4>>(); }

template <class C>
static hipError_t launch_tile(const uint8_t *x, const float *token_scale, const uint8_t *w, int64_t M, int64_t N, int64_t K, int64_t groups, int64_t per,
                              const float *scales, void *y, int y_type, hipStream_t s)
{
    const int64_t tiles_m = (M + C::BM - 1) / C::BM, tiles_n = (N + C::BN - 1) / C::BN;
    if (tiles_m * tiles_n > (int64_t)0xffffffff / C::THREADS) return hipErrorInvalidConfiguration;
    const DeviceInfo *info;
    const hipError_t e = device_info(&info);      // the tiles' LDS is an attribute of the kernels, set once per device
    if (e != hipSuccess) return e;
    grouped_tile_kernel<C><<<dim3((unsigned)(tiles_m * tiles_n)), dim3(C::THREADS), C::LDS_BYTES, s>>>(x, w, scales, (int)M, (int)N, (int)k_tiles(K), (int)tiles_m,
                                                                                                       (int)tiles_n, (uint32_t)per, reciprocal((uint32_t)per),
                                                                                                       (int)groups, token_scale, y, y_type);
    return hipGetLastError();
}

hipError_t launch_grouped_linear(const uint8_t *x, const float *token_scale, const uint8_t *w, int64_t M, int64_t N, int64_t K, int64_t group, const float *scales,
                                 void *y, int y_type, hipStream_t s)
{
    const int64_t kt = k_tiles(K), groups = (K + group - 1) / group, per = group > KT ? min(group / KT, kt) : 1;
    if (M > 64) {
        const bool large = ((M + 255) / 256) * ((N + 255) / 256) >= 200;
#define FPTQ_TILE(GT)                                                                                                             \
    do {                                                                                                                          \
        if (large) return launch_tile<Large<GT>>(x, token_scale, w, M, N, K, groups, per, scales, y, y_type, s);                  \
        return launch_tile<Small<GT>>(x, token_scale, w, M, N, K, groups, per, scales, y, y_type, s);                             \
    } while (0)
        if (group == 32) FPTQ_TILE(4);
        if (group == 64) FPTQ_TILE(2);
        FPTQ_TILE(1);
#undef FPTQ_TILE
    }
#define FPTQ_FEW(MT, GT)                                                                                                                   \
    do {                                                                                                                                   \
        grouped_few_kernel<8, 1, MT, 1, GT><<<dim3((unsigned)((N + 15) / 16), (unsigned)((M + 16 * MT - 1) / (16 * MT))), dim3(512), 0, s>>>(   \
            x, w, scales, (int)M, (int)N, (int)kt, (int)groups, (uint32_t)per, reciprocal((uint32_t)per), token_scale, y, y_type);         \
        return hipGetLastError();                                                                                                          \
    } while (0)
#define FPTQ_FEW_GT(GT)              \
    do {                             \
        if (M <= 16) FPTQ_FEW(1, GT); \
        FPTQ_FEW(4, GT);             \
    } while (0)
    if (group == 32) FPTQ_FEW_GT(4);
    if (group == 64) FPTQ_FEW_GT(2);
    FPTQ_FEW_GT(1);
#undef FPTQ_FEW_GT
#undef FPTQ_FEW
}

}  // namespace fptq
