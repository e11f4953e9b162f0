// Causal attention over whole prompts, packed one after the other, with grouped heads.
//
//   o = sum_t p_t v_t / sum_t p_t,   p_t = exp2(c (q . k_t) - m),   c = scale * log2 e,   m the running maximum of c (q . k_t)
//
// in one pass over the keys: bound by the matrix cores and, next to them, by the exponentials.  A workgroup takes 128 tokens of a query head, a wave 32 of
// them, as columns: S^T = K Q^T and O^T = V^T P^T with 32 x 32 x 16 products.  So a lane holds scores of one token only (half of them, the lane 32
// away the others), the softmax needs one exchange where a maximum has grown, and what S^T leaves in a lane is what O^T wants of it: keys
// 4 h + e and 8 + 4 h + e of every 16, h the half of the wave.  Keys and values go to LDS 64 tokens at a time without passing through registers,
// two tiles deep; values are read back transposed by the LDS.  16-byte granules are exchanged within rows so that these reads have no bank conflicts; the
// exchange is made by the addresses that the copies' lanes read from.  Scores of a tile are made while the weights of the tile before are, and their
// maximum beside that tile's products, so that matrix instructions run under the others.
//
// P is rounded to bf16 (half a step, 2^-8 of each term); maxima, sums and outputs are fp32.  The accumulators are rescaled only when a maximum has grown by
// more than 2^8: until then p is at most 256 and loses nothing, being a float.
//
// Measured (a call among others, on several cards; the kernel under the profiler's trace, two batches in turn): 8192 tokens, 64 heads over 8 of 128: 960 to 1005 us; 997
// to 1022, 1080 to 1145 TFLOP/s, where a library product of 8192 x 8192 x 8192 reaches 1130 to 1270.  1.69 million cycles, matrix cores busy 63 % of them, at
// 1.7 GHz: with zeros for data, which draw less power, 750 us.  4096 tokens, 32 heads over 8: 131 to 145 us; 142 to 150.  Nine prompts of 6000 tokens together, 32
// heads over 32: 78 to 91 us; 72 to 77.  With 64 values a head, 32 heads over 8, 4096 and 8192 tokens: 82 and 293 us, where the operations take 61 and 244.
// A workgroup costs 10000 to 13000 cycles besides its tiles (about 1450 each, two workgroups a CU): 5000 to 7000 until the first tile is there, 3000 at the
// diagonal, 1700 to write.  So a prompt that leaves CUs idle is as long as its last block's chain: 512, 1024 and 2048 tokens, 32 heads over 8 of 128, 12.4, 21 and 45 us.
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
constexpr int AHEAD = 4;                       // products whose operands are read from LDS before the first one (2, 3 and 6: the same within 1 %)
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

// 16 bytes a lane from memory to LDS, which is written in the order of the lanes, from `to` on.  As assembly, because the compiler, which cannot tell tiles apart,
// would wait for the tile on its way before it reads the one that is there, every time (8192 tokens, 64 heads: 1096 us); it has no outputs, and what it
// writes is waited for at the barrier, by s_waitcnt vmcnt(0).
__device__ inline void copy_to_lds(v4i descriptor, uint32_t to, uint32_t offset)
{
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(to), "v"(offset), "s"(descriptor) : "memory");
}
// raw buffer descriptor; reads past its end are zeros
__device__ inline v4i descriptor_of(const void *base, int bytes)
{
    const uint64_t p = (uint64_t)base;
    return v4i{uniform((int)p), uniform((int)(p >> 32) & 0xffff), uniform(bytes), RSRC_FLAGS};
}
__device__ inline uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)LDS_PTR((void *)p); }

// bf16 pairs that hold an infinity or a NaN, as 0xffff each; whether a pair does, in bits 15 and 31
__device__ inline uint32_t not_finite(uint32_t w)
{
    const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
    return lo | hi;
}
__device__ inline uint32_t exponent_carry(uint32_t w) { return (w & 0x7f807f80u) + 0x00800080u; }

// What a workgroup does: QT tokens of a head.  Items of the longest sequence come first and a sequence's last tokens first: what ends last is short, and
// blocks that read the same keys and values run at about the same time (ordered by their own lengths each reads them from memory again).  More than
// SORTED sequences are taken in their own order.
struct Item {
    int begin, n, row0, head;                  // n 0: there is none
};
struct Items {
    static constexpr int SORTED = 32;
    const PromptArgs &a;
    Span own;                                  // the lane's sequence, its blocks and the blocks that come before them
    int blocks, before;
    __device__ explicit Items(const PromptArgs &args) : a(args), own{0, 0}, before(0)
    {
        const int lane = lane_id();
        if (lane < a.seq.count) own = new_tokens(a.seq, lane);
        blocks = (own.n + QT - 1) / QT;
        const int order = blocks * 64 + 63 - lane;       // of two with as many blocks the first one comes first; 2^17 blocks at most
        if (a.seq.count <= SORTED)
            for (int j0 = 0; j0 < a.seq.count; j0 += 8)  // eight at a time: one by one each waits for the one before, 180 cycles
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int other = __builtin_amdgcn_readlane(order, j0 + j);
                    before += other > order ? other >> 6 : 0;
                }
    }
    __device__ Item at(int index) const
    {
        const int block = index / a.heads, slot = index % a.heads;
        Item i = {0, 0, 0, slot};
        if (a.heads % 8 == 0) i.head = slot % 8 * (a.heads / 8) + slot / 8;      // an XCD, every eighth workgroup, gets heads that share keys and values
        int place;                                     // from the sequence's last block on
        if (a.seq.count <= SORTED) {
            const uint64_t hit = __ballot(block >= before && block < before + blocks);
            if (!hit) return i;
            const int b = __builtin_ctzll(hit);
            place = block - __builtin_amdgcn_readlane(before, b);
            i.begin = __builtin_amdgcn_readlane(own.begin, b), i.n = __builtin_amdgcn_readlane(own.n, b);
        } else {
            const Found f = find_sequence(a.seq.count, block, [&](int b) { return (new_tokens(a.seq, b).n + QT - 1) / QT; });
            if (f.sequence < 0) return i;
            const Span span = new_tokens(a.seq, uniform(f.sequence));
            place = uniform(f.place), i.begin = uniform(span.begin), i.n = uniform(span.n);
        }
        i.row0 = ((i.n + QT - 1) / QT - 1 - place) * QT;
        return i;
    }
};

template <int N>
struct Halves {
    static constexpr int value = N;
};

template <int D>
__global__ __launch_bounds__(256, 2) void prompt_attention_kernel(const int32_t *cu, int32_t count, int32_t tokens, int32_t heads, int32_t group,
                                                                 const PromptArgs rest)
{
    // what a workgroup needs first comes with the dispatch
    PromptArgs a = rest;
    a.seq.cu = cu, a.seq.count = count, a.seq.tokens = tokens, a.heads = heads, a.group = group;
    constexpr int KS = D / 16, DB = D / 32, ROW = D * 2, TILE = KTILE * ROW, GRANULES = D / 8;
    constexpr int COPIES = TILE / 1024 / 4, ROWS_PER_COPY = 1024 / ROW;        // a copy: 1 KB, 16 bytes a lane
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2][2][TILE];         // [stage][keys, values]
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), col = lane & 31, half = lane >> 5;

    const Item item = Items(a).at(blockIdx.x);
    if (!item.n) return;
    const int begin = item.begin, n = item.n, row0 = item.row0, head = item.head;
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
    const uint32_t to = uniform(lds_address(lds) + wave * COPIES * 1024);
    // rows past the sequence's end are beyond the descriptor's and arrive as zeros
    const auto fill_keys = [&](int tile, int stage) {
        const v4i r = descriptor_of(k_base + (int64_t)tile * KTILE * k_row, (min(n - tile * KTILE, KTILE) - 1) * (int)k_row + ROW);
#pragma unroll
        for (int c = 0; c < COPIES; ++c) copy_to_lds(r, to + stage * 2 * TILE + c * 1024, k_off[c]);
    };
    const auto fill_values = [&](int tile, int stage) {
        const v4i r = descriptor_of(v_base + (int64_t)tile * KTILE * v_row, (min(n - tile * KTILE, KTILE) - 1) * (int)v_row + ROW);
#pragma unroll
        for (int c = 0; c < COPIES; ++c) copy_to_lds(r, to + stage * 2 * TILE + TILE + c * 1024, v_off[c]);
    };

    // where the lane reads: of keys granule 2 k + half of row col; of values four tokens a read, 4 half + t / 4 of eight, values 32 d + 16 part + 4 (t % 4) ..,
    // of which it gets its own of each token
    const int t = lane & 15, part = lane >> 4 & 1;
    uint32_t k_at[KS], v_at[DB];
#pragma unroll
    for (int k = 0; k < KS; ++k) k_at[k] = col * ROW + key_granule<D>(col, 2 * k + half) * 16;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        const int r = 4 * half + (t >> 2), v = 32 * d + 16 * part + 4 * (t & 3);
        v_at[d] = r * ROW + value_granule<D>(r, v / 8) * 16 + v % 8 * 2;
    }

    constexpr Halves<2> ALL;
    v16f o[DB] = {};
    float m = NONE, l = 0.0f;
    // scores of the tile in `stage`
    const auto scores = [&](int stage, v16f(&s)[2]) {
        const uint8_t *const keys = lds[stage][0];
        s[0] = v16f{}, s[1] = v16f{};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, *(const v4u *)(keys + k_at[k] + b * 32 * ROW)), q[k], s[b], 0, 0, 0);
    };
    // of the tile's first 32 keys, or of all
    const auto largest = [&](auto halves, const v16f(&s)[2]) {
        float top = s[0][0];
#pragma unroll
        for (int e = 1; e < 16 * halves.value; ++e) top = fmaxf(top, s[e >> 4][e & 15]);
        return top * a.scale;
    };
    const auto raise = [&](float top) {
        if (__any(top > m + 8.0f)) {
            const float grown = fmaxf(m, other_half_max(top));
            const float by = m == NONE ? 0.0f : __builtin_amdgcn_exp2f(m - grown);
            m = grown;
            l *= by;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] *= by;
        }
    };
    // weights of 16 keys each, as the products want them
    const auto weights = [&](auto halves, const v16f(&s)[2], v8bf(&p)[4]) {
        const float base = m == NONE ? 0.0f : m;
#pragma unroll
        for (int k = 0; k < 2 * halves.value; ++k) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k >> 1][8 * (k & 1) + 2 * e], a.scale, -base));
                const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k >> 1][8 * (k & 1) + 2 * e + 1], a.scale, -base));
                l += x + y;
                w[e] = pack_bf16(x, y);
            }
            p[k] = __builtin_bit_cast(v8bf, v4u{w[0], w[1], w[2], w[3]});
        }
    };
    const auto value_fragment = [&](int stage, int d, int k) {
        const uint8_t *const from = lds[stage][1] + v_at[d] + k * 16 * ROW;
        const uint2 x = read_column(from), y = read_column(from + 8 * ROW);
        return v4u{x.x, x.y, y.x, y.y};
    };

    const auto products = [&](auto halves, int stage, const v8bf(&p)[4]) {
#pragma unroll
        for (int k = 0; k < 2 * halves.value; ++k)
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, value_fragment(stage, d, k)), p[k], o[d], 0, 0, 0);
    };

    // A wave's last tile is the one with its own tokens, the only one with keys that some of its rows do not see.  Until then scores of a tile are made
    // while the weights of the tile before are, and their maximum beside that tile's products: matrix instructions run under the others.
    const int tiles = (min(row0 + QT, n) + KTILE - 1) / KTILE, own = min(tiles, first / KTILE + 1);
    const auto turn = [&](int tile, int stage) {             // what all waves do before tile `tile`: its values and the next one's keys are there
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        __syncthreads();
        if (tile + 2 < tiles) fill_keys(tile + 2, stage);
        if (tile + 1 < tiles) fill_values(tile + 1, stage ^ 1);
    };
    fill_keys(0, 0);
    fill_values(0, 0);
    if (tiles > 1) fill_keys(1, 1);
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    __syncthreads();
    if (first >= n) {                                        // none of the wave's rows is there: it copies for the others
        for (int tile = 0; tile < tiles; ++tile) turn(tile, tile & 1);
        return;
    }
    v16f s[2], later[2];
    scores(0, s);
    float top = largest(ALL, s);
    const auto step = [&](int tile, int stage, const v16f(&now)[2], v16f(&next)[2]) {
        turn(tile, stage);
        raise(top);
        __builtin_amdgcn_sched_barrier(0);
        v8bf p[4];
        scores(stage ^ 1, next);
        weights(ALL, now, p);
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 112 / (2 * KS), 0);
        }
        asm volatile("" : "+v"(l));                           // here and not after the barrier, where nothing runs under it
        __builtin_amdgcn_sched_barrier(0);
        products(ALL, stage, p);
        top = largest(ALL, next);
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * AHEAD, 0);
#pragma unroll
        for (int i = 0; i < 4 * DB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 32 / (4 * DB), 0);
        }
        asm volatile("" : "+v"(top));
        __builtin_amdgcn_sched_barrier(0);
    };
    int tile = 0;
    for (; tile + 2 < own; tile += 2) {
        step(tile, 0, s, later);
        step(tile + 1, 1, later, s);
    }
    if (tile + 1 < own) {
        step(tile, 0, s, later);
        s[0] = later[0], s[1] = later[1];
        ++tile;
    }
    {
        const int stage = tile & 1, key0 = tile * KTILE, halves = (first / 32 & 1) + 1;
        turn(tile, stage);
        // The wave's own 32 tokens are the last or the first half of the tile, and what is behind them nobody sees.
        v8bf p[4];
        uint32_t carry = 0;                                   // of any of their values that is not finite
        const auto last = [&](auto halves) {
            constexpr int own_half = halves.value - 1;
#pragma unroll
            for (int c = 0; c < TILE / 2048; ++c) {
                const v4u w = *(const v4u *)(lds[stage][1] + own_half * (TILE / 2) + c * 1024 + lane * 16);
                carry |= exponent_carry(w[0]) | exponent_carry(w[1]) | exponent_carry(w[2]) | exponent_carry(w[3]);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if ((e >> 2) * 8 + half * 4 + (e & 3) > col) s[own_half][e] = NONE;
            raise(largest(halves, s));
            weights(halves, s, p);
            asm volatile("" : "+v"(l));                       // its terms are summed here and not kept until the end
            carry = __any((carry & 0x80008000u) != 0);
            if (!carry) products(halves, stage, p);
        };
        if (halves == 2) last(Halves<2>());
        else last(Halves<1>());
        if (carry) {
            // An infinity or NaN that only some of the rows see would reach the others as 0 times itself.  It is taken out, and what it makes of the
            // rows that see it is found by products of indicators: NaN counts as both infinities.
#pragma unroll 1
            for (int k = 0; k < 2 * halves; ++k) {
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    v4u w = value_fragment(stage, d, k), up, down, see;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + 16 * k + (e >> 1) * 8 + half * 4 + 2 * (e & 1);
                        see[e] = (key <= row ? 0x3f80u : 0u) | (key + 1 <= row ? 0x3f800000u : 0u);
                        const uint32_t bad = not_finite(w[e]), negative = (w[e] & 0x8000u ? 0xffffu : 0u) | (w[e] & 0x80000000u ? 0xffff0000u : 0u);
                        const uint32_t nan = (w[e] & 0x7fu ? 0xffffu : 0u) | (w[e] & 0x7f0000u ? 0xffff0000u : 0u);
                        up[e] = bad & (~negative | nan) & 0x3f803f80u, down[e] = bad & (negative | nan) & 0x3f803f80u;
                        w[e] &= ~bad;
                    }
                    const v16f zero = {};
                    const v16f ups = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, up), __builtin_bit_cast(v8bf, see), zero, 0, 0, 0);
                    const v16f downs = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, down), __builtin_bit_cast(v8bf, see), zero, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        if (ups[e] > 0.0f) o[d][e] += __builtin_inff();
                        if (downs[e] > 0.0f) o[d][e] -= __builtin_inff();
                    }
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, w), p[0], o[d], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
                p[0] = p[1], p[1] = p[2], p[2] = p[3];
            }
        }
    }
    while (++tile < tiles) turn(tile, tile & 1);             // the waves of later tokens go on
    // The lane holds values 8 i + 4 half .. of its row; halves exchange fours, so that each stores eight in a row.
    const float sum = other_half_sum(l), r = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint16_t *const out = a.out + ((int64_t)(begin + row) * a.heads + head) * D + half * 8;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack_bf16(o[d][8 * e + 2 * i] * r, o[d][8 * e + 2 * i + 1] * r);
            const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
            if (row < n) *(v4u *)(out + d * 32 + e * 16) = v4u{x[0], y[0], x[1], y[1]};
        }
}

hipError_t launch_prompt_attention(Heads q, Heads k, Heads v, const Sequences &s, int heads, int kv_heads, int head_dim, float scale, uint16_t *out,
                                   hipStream_t stream)
{
    const PromptArgs a = {q, k, v, s, out, heads, heads / kv_heads, scale * 1.44269504088896341f};
    int64_t blocks = s.tokens / QT + (int64_t)s.count;               // of n tokens: n / QT + 1 at most
    if (blocks > s.tokens) blocks = s.tokens;
    if (blocks * heads > 1 << 23) return hipErrorInvalidConfiguration;      // before the device is asked for anything
    const DeviceInfo *info;
    hipError_t e = device_info(&info);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)(blocks * heads));
    if (head_dim == 128) prompt_attention_kernel<128><<<grid, dim3(256), 0, stream>>>(s.cu, s.count, s.tokens, heads, a.group, a);
    else prompt_attention_kernel<64><<<grid, dim3(256), 0, stream>>>(s.cu, s.count, s.tokens, heads, a.group, a);
    return hipGetLastError();
}

}  // namespace fptq
