// Causal attention over whole prompts, packed one after the other, with grouped heads.
//
//   o = sum_t p_t v_t / sum_t p_t,   p_t = exp2(c (q . k_t) - m),   c = scale * log2 e,   m the running maximum of c (q . k_t)
//
// in one pass over the keys: bound by the matrix cores and, next to them, by the exponentials.  A workgroup takes 128 tokens of a query head, a wave 32 of
// them, as columns: S^T = K Q^T and O^T = V^T P^T with 32 x 32 x 16 products.  So a lane holds scores of one token only (half of them, the lane 32
// away the others), the softmax needs one exchange where a maximum has grown, and what S^T leaves in a lane is what O^T wants of it: keys
// 4 h + e and 8 + 4 h + e of every 16, h the half of the wave.  Keys and values go to LDS 64 tokens at a time without passing through registers,
// two tiles deep; values are read back transposed by the LDS.  16-byte granules are exchanged within rows so that these reads have no bank conflicts; the exchange is
// made by the addresses that the copies' lanes read from.
//
// P is rounded to bf16 (half a step, 2^-9 of each term); maxima, sums and outputs are fp32.  The accumulators are rescaled only when a maximum has grown by
// more than 2^8: until then p is at most 256 and loses nothing, being a float.
#include "fptq_attention.h"

namespace fptq {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

struct PromptArgs {
    Heads q, k, v;
    Sequences seq;
    uint16_t *out;
    int heads, group;
    float scale;                               // times log2 e
};

constexpr float NONE = -__builtin_inff();
constexpr int QT = 128, KTILE = 64;            // tokens of a workgroup, keys of a tile

__device__ inline float other_half_max(float v)
{
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ inline float other_half_sum(float v)
{
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Where granule g (16 bytes) of a row lies in LDS.  Keys are read by 32 rows at the same granule, values by 4 rows at 4 neighbouring ones.
template <int D>
__device__ inline int key_granule(int row, int g) { return D == 128 ? g ^ (row & 15) : g ^ (row >> 1 & 7); }
template <int D>
__device__ inline int value_granule(int row, int g) { return D == 128 ? g ^ ((row & 3) << 2) : g ^ ((row >> 1 & 1) << 2); }

// four rows' values, 16 bits each, of the lane's column: of 16 lanes' addresses four in a row point to a row's 16 columns
__device__ inline uint2 read_column(const uint8_t *p)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(p)));
}

// 16 bytes a lane from memory to LDS, which is written in the order of the lanes
__device__ inline void copy_to_lds(__amdgpu_buffer_rsrc_t r, uint8_t *to, uint32_t offset) { __builtin_amdgcn_raw_ptr_buffer_load_lds(r, LDS_PTR(to), 16, offset, 0, 0, 0); }

// bf16 pairs that hold an infinity or a NaN, as 0xffff each
__device__ inline uint32_t not_finite(uint32_t w)
{
    const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
    return lo | hi;
}

// Blocks of QT tokens by the work in them, the most first: of every sequence long enough its block at one place, then the blocks one place before.
// Workgroups begin in this order, so the last to end are short (nine prompts of 6000 tokens together: in the sequences' own order 99 us, so 78).
struct Block {
    int sequence, place;
};
__device__ inline int blocks_of(const Sequences &s, int b) { return b < s.count ? (new_tokens(s, b).n + QT - 1) / QT : 0; }
__device__ inline Block find_block(const Sequences &s, int item)
{
    const int first = blocks_of(s, lane_id());
    if (s.count == 1) {
        const int place = __builtin_amdgcn_readlane(first, 0) - 1 - item;
        return {place < 0 ? -1 : 0, place};
    }
    // a sum over the sequences
    const auto over_all = [&](auto of) {
        int sum = of(first);
        for (int b0 = 64; b0 < s.count; b0 += 64) sum += of(blocks_of(s, b0 + lane_id()));
        return __builtin_amdgcn_readlane(wave_prefix(sum), 63);
    };
    const auto from_on = [&](int place) { return over_all([=](int n) { return max(n - place, 0); }); };      // blocks at this place or behind it
    if (item >= from_on(0)) return {-1, 0};
    int place = 0, above = 1;                         // the last place that has item or fewer blocks behind it
    while (item < from_on(above)) place = above, above *= 2;
    while (above - place > 1) {
        const int middle = (place + above) / 2;
        if (item < from_on(middle)) place = middle;
        else above = middle;
    }
    const Found f = find_sequence(s.count, item - from_on(place + 1), [&](int b) { return (b < 64 ? first : blocks_of(s, b)) > place ? 1 : 0; });
    return {f.sequence, place};
}

template <int D>
__global__ __launch_bounds__(256, 2) void prompt_attention_kernel(const PromptArgs a)
{
    constexpr int KS = D / 16, DB = D / 32, ROW = D * 2, TILE = KTILE * ROW, GRANULES = D / 8;
    constexpr int COPIES = TILE / 1024 / 4, ROWS_PER_COPY = 1024 / ROW;        // a copy: 1 KB, 16 bytes a lane
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2][2][TILE];         // [stage][keys, values]
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), col = lane & 31, half = lane >> 5;

    // workgroups: heads within blocks of tokens; the XCDs (every eighth workgroup) get heads that share keys and values
    const int block = blockIdx.x / a.heads, slot = blockIdx.x % a.heads;
    const int head = a.heads % 8 == 0 ? slot % 8 * (a.heads / 8) + slot / 8 : slot;
    const Block f = find_block(a.seq, block);
    if (f.sequence < 0) return;
    const Span span = new_tokens(a.seq, uniform(f.sequence));
    const int begin = uniform(span.begin), n = uniform(span.n);
    const int row0 = uniform(f.place) * QT;
    const int first = row0 + wave * 32, row = first + col;

    v8bf q[KS];
    {
        const uint16_t *const from = a.q.p + (int64_t)(begin + min(row, n - 1)) * a.q.token + (int64_t)head * a.q.head + half * 8;
#pragma unroll
        for (int k = 0; k < KS; ++k) q[k] = __builtin_bit_cast(v8bf, *(const v4u *)(from + k * 16));
    }

    const int64_t k_row = a.k.token * 2, v_row = a.v.token * 2;
    const uint8_t *const k_base = (const uint8_t *)(a.k.p + (int64_t)begin * a.k.token + (int64_t)(head / a.group) * a.k.head);
    const uint8_t *const v_base = (const uint8_t *)(a.v.p + (int64_t)begin * a.v.token + (int64_t)(head / a.group) * a.v.head);
    uint32_t k_off[COPIES], v_off[COPIES];
#pragma unroll
    for (int c = 0; c < COPIES; ++c) {
        const int r = (wave * COPIES + c) * ROWS_PER_COPY + lane / GRANULES, g = lane % GRANULES;
        k_off[c] = r * (uint32_t)k_row + key_granule<D>(r, g) * 16, v_off[c] = r * (uint32_t)v_row + value_granule<D>(r, g) * 16;
    }
    // rows past the sequence's end are beyond the descriptor's and arrive as zeros
    auto fill = [&](int tile, int stage) {
        const int left = min(n - tile * KTILE, KTILE);
        const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc((void *)(k_base + (int64_t)tile * KTILE * k_row), 0, (left - 1) * (int)k_row + ROW, RSRC_FLAGS);
        const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc((void *)(v_base + (int64_t)tile * KTILE * v_row), 0, (left - 1) * (int)v_row + ROW, RSRC_FLAGS);
#pragma unroll
        for (int c = 0; c < COPIES; ++c) {
            copy_to_lds(kr, &lds[stage][0][(wave * COPIES + c) * 1024], k_off[c]);
            copy_to_lds(vr, &lds[stage][1][(wave * COPIES + c) * 1024], v_off[c]);
        }
    };

    v16f o[DB] = {};
    float m = NONE, base = 0.0f, l = 0.0f;
    const int tiles = (min(row0 + QT, n) + KTILE - 1) / KTILE;
    fill(0, 0);
    for (int tile = 0; tile < tiles; ++tile) {
        const int stage = tile & 1;
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        __syncthreads();
        if (tile + 1 < tiles) fill(tile + 1, stage ^ 1);
        const int key0 = tile * KTILE;
        if (key0 > first + 31) continue;                     // beyond all of the wave's rows
        v16f s[2] = {};
        const uint8_t *const keys = lds[stage][0], *const values = lds[stage][1];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int r = b * 32 + col;
                const v4u x = *(const v4u *)(keys + r * ROW + key_granule<D>(r, 2 * k + half) * 16);
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, x), q[k], s[b], 0, 0, 0);
            }
        const bool diagonal = key0 + KTILE - 1 > first;
        if (diagonal) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (key0 + b * 32 + (e >> 2) * 8 + half * 4 + (e & 3) > row) s[b][e] = NONE;
        }
        float top = s[0][0];
#pragma unroll
        for (int e = 1; e < 32; ++e) top = fmaxf(top, s[e >> 4][e & 15]);
        top *= a.scale;
        if (__any(top > m + 8.0f)) {
            const float grown = fmaxf(m, other_half_max(top));
            const float by = m == NONE ? 0.0f : __builtin_amdgcn_exp2f(m - grown);
            m = grown, base = grown == NONE ? 0.0f : grown;
            l *= by;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] *= by;
        }
        v8bf p[4];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][8 * h + 2 * e], a.scale, -base));
                    const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][8 * h + 2 * e + 1], a.scale, -base));
                    l += x + y;
                    w[e] = pack_bf16(x, y);
                }
                p[2 * b + h] = __builtin_bit_cast(v8bf, v4u{w[0], w[1], w[2], w[3]});
            }
        const int t = lane & 15, part = lane >> 4 & 1;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // four tokens a read: 16 k + 8 j + 4 half + t / 4, values 32 d + 16 part + 4 (t % 4) ..; the lane gets its own value of each
                uint2 x[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int r = 16 * k + 8 * j + 4 * half + (t >> 2), v = 32 * d + 16 * part + 4 * (t & 3);
                    x[j] = read_column(values + r * ROW + value_granule<D>(r, v / 8) * 16 + v % 8 * 2);
                }
                v4u w = {x[0].x, x[0].y, x[1].x, x[1].y};
                if (diagonal) {
                    // An infinity or NaN that only some of the rows see would reach the others as 0 times itself.  It is taken out, and what it makes of the
                    // rows that see it is found by products of indicators: NaN counts as both infinities.
                    v4u bad;
#pragma unroll
                    for (int e = 0; e < 4; ++e) bad[e] = not_finite(w[e]);
                    if (__any((bad[0] | bad[1] | bad[2] | bad[3]) != 0)) {
                        v4u up, down, see;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = key0 + 16 * k + (e >> 1) * 8 + half * 4 + 2 * (e & 1);
                            see[e] = (key <= row ? 0x3f80u : 0u) | (key + 1 <= row ? 0x3f800000u : 0u);
                            const uint32_t negative = (w[e] & 0x8000u ? 0xffffu : 0u) | (w[e] & 0x80000000u ? 0xffff0000u : 0u);
                            const uint32_t nan = (w[e] & 0x7fu ? 0xffffu : 0u) | (w[e] & 0x7f0000u ? 0xffff0000u : 0u);
                            up[e] = bad[e] & (~negative | nan) & 0x3f803f80u, down[e] = bad[e] & (negative | nan) & 0x3f803f80u;
                            w[e] &= ~bad[e];
                        }
                        const v16f zero = {};
                        const v16f ups = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, up), __builtin_bit_cast(v8bf, see), zero, 0, 0, 0);
                        const v16f downs = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, down), __builtin_bit_cast(v8bf, see), zero, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            if (ups[e] > 0.0f) o[d][e] += __builtin_inff();
                            if (downs[e] > 0.0f) o[d][e] -= __builtin_inff();
                        }
                    }
                }
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, w), p[k], o[d], 0, 0, 0);
            }
    }
    const float sum = other_half_sum(l), r = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (row < n) {
        uint16_t *const to = a.out + ((int64_t)(begin + row) * a.heads + head) * D + half * 4;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *(uint2 *)(to + d * 32 + e * 8) = uint2{pack_bf16(o[d][4 * e] * r, o[d][4 * e + 1] * r), pack_bf16(o[d][4 * e + 2] * r, o[d][4 * e + 3] * r)};
    }
}

hipError_t launch_prompt_attention(Heads q, Heads k, Heads v, const Sequences &s, int heads, int kv_heads, int head_dim, float scale, uint16_t *out,
                                   hipStream_t stream)
{
    const DeviceInfo *info;
    hipError_t e = device_info(&info);
    if (e != hipSuccess) return e;
    const PromptArgs a = {q, k, v, s, out, heads, heads / kv_heads, scale * 1.44269504088896341f};
    int64_t blocks = s.tokens / QT + (int64_t)s.count;               // of n tokens: n / QT + 1 at most
    if (blocks > s.tokens) blocks = s.tokens;
    if (blocks * heads > 1 << 23) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)(blocks * heads));
    if (head_dim == 128) prompt_attention_kernel<128><<<grid, dim3(256), 0, stream>>>(a);
    else prompt_attention_kernel<64><<<grid, dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace fptq
