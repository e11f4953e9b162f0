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

hipError_t launch_grouped_linear(const uint8_t *x, const float *token_scale, const uint8_t *w, int64_t M, int64_t N, int64_t K, int64_t group, const float *scales,
                                 void *y, int y_type, hipStream_t s)
{
    const int64_t kt = k_tiles(K), groups = (K + group - 1) / group, per = group > KT ? group / KT : 1;
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
