// Attention over the paged 8-bit cache: a sequence's last tokens (one each in a token loop) against all its keys and values.
//
//   o = sum_t p_t v_t / sum_t p_t,   p_t = exp2(c (q . k_t) - m),   c = scale * log2 e,   m the running maximum of c (q . k_t)
//
// in one pass over the cache.  What bounds it is the reading of the cache: 2 D bytes a token and kv head, some 2 G operations a byte.
//
// A wave takes a page-head (64 tokens of a kv head) at a time.  The query rows that read it (G heads of every new token) are the columns of the matrix
// instructions, 16 of them or 32:  S^T = K Q^T and O^T = V^T P^T.  Where the rows fit one such tile nothing of the cache is read twice; of more rows (a group of 40,
// a chunk of a prompt behind what is cached of it) every tile reads and widens it for itself.  Codes go from memory to registers 16 bytes a
// lane and are widened to bf16 there, scale included (both exact), two values an instruction; the page's layout is such that each lane's 16 bytes are
// what the instructions want of it: of keys 16 values of one token; of values the 16 tokens whose scores the lane holds, when row
// 4 g + i of the b-th 16 of S^T is token 16 g + 4 b + i.  So P^T needs no exchange between lanes and nothing goes through LDS in the loop.
//
// P is rounded to bf16 (half a step, 2^-8 of each term); maxima, sums and outputs are fp32.  The accumulators are rescaled only when a maximum has
// grown by more than 2^8: until then p is at most 256 and loses nothing, being a float.
//
// Ragged batches: a unit is a sequence, kv head and 16 or 32 rows.  Units of more than two shares of all pages are cut into equal parts, whose
// results a second kernel joins.  Everything about lengths is read on the device, so a captured launch serves growing sequences.
//
// Measured: 64 sequences of up to 32768 tokens (64 heads over 8, 2.72 GB of codes) 476 us, 5.7 TB/s where a kernel that only reads takes 440 to 454; 32 of up to 4096
// (163 MB) 36.9 to 38.2 us, reading alone 27.5; short calls are a chain of memory latencies (length, page number, codes): a token behind 333 6.6 us, and 9.0 with a table
// of 4096 pages, for which the join is launched.  256 new tokens, the last of 8192, 32 heads over 8 of 128, 57 us, 1024 of them 148, where the operations take 30 and 114.
#include "fptq_attention.h"

namespace fptq {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

// Waves of a workgroup, which take its pages in turn.  Eight share a unit's pages out further: 32 sequences of up to 4096 tokens, 16 rows, 36.9 us, with
// four waves 41.1; 64 of up to 32768 475 and 507.  With 32 rows four are faster, each with more pages for what a wave costs at its beginning and end:
// 4 tokens behind 131072 20.8 us, with eight 22.4.  (Loading two pages ahead instead of one: 21.5 and 23.9.)
__host__ __device__ constexpr int waves_of(int row_tiles) { return row_tiles == 2 ? 4 : 8; }

// Pages of a part at least.  A wave alone on its SIMD takes 2 us a page, what a part costs besides and the join 6 (a token behind 4096, 8 kv heads: 23.0 us
// uncut, 13.6 in parts of 8 pages).  Where there are 32 pages for every compute unit, parts are no smaller than that (4 tokens behind 131072:
// 20.0 us, parts of 16 pages 24.7).  Nor where there are units for every compute unit: cutting then only evens out their lengths (32
// sequences of up to 64 pages, 8 kv heads: 36.9 us uncut, 45.9 with those of more than 48 cut).
constexpr int LEAST_SHARE = 8, FULL_SHARE = 32;
static int least_share(int64_t units) { return units >= DEFAULT_CUS ? FULL_SHARE : LEAST_SHARE; }
constexpr int PARTS = 1536;        // what very many pages are shared out to (64 sequences of up to 32768 tokens, the only shape timed, 478 us; 1280 483, 1024 507, 2048 490, 1792 499)
constexpr int MAX_GRID = 1024;     // workgroups; they go on from part to part, so that room in the table for many more parts costs little
constexpr int JOIN_WAVES = 8;      // of a workgroup of the join
constexpr int JOINED = 512;        // units that the join's grid is for; if more are cut, its workgroups take several

struct DecodeArgs {
    Heads q;
    Sequences seq;
    Cache cache;
    uint16_t *out;
    float *parts;                              // [2 PARTS][rows][D] sums, then [2 PARTS][rows][2] maxima and weights
    int heads, kv_heads, group;
    float scale;                               // times log2 e
    int most_items;                            // parts and whole units there can be
    int least_share;
};

struct Shape {
    int tiles, pages;                          // of a sequence: row tiles of each kv head, pages
};
template <int ROWS>
__device__ inline Shape shape_of(const DecodeArgs &a, int b)
{
    if (b >= a.seq.count) return {0, 0};
    const int rows = new_tokens(a.seq, b).n * a.group;
    return {(rows + ROWS - 1) / ROWS, (int)min((int64_t)(length_of(a.seq, b) + PAGE - 1) / PAGE, a.seq.table_width)};
}

// How the pages are shared out: units of more than twice `most` pages, a share of all, are cut into equal parts of at most that.
// (Cutting those of up to twice as many costs the join's 5 us and balances little.)  Every wave finds this out for itself, 64 sequences at a time; the
// shapes of the first 64 stay in its lanes.
template <int ROWS>
struct Shares {
    const DecodeArgs &a;
    Shape first;
    int most, items;                           // parts and whole units in all
    bool any;                                  // whether any unit is cut
    __device__ explicit Shares(const DecodeArgs &args) : a(args), first{0, 0}, most(1 << 29), any(false)
    {
        const int whole = a.seq.count * ((a.group + ROWS - 1) / ROWS) * a.kv_heads;      // units of sequences of one token
        items = whole;
        if (!a.parts && !a.seq.cu) return;     // it takes no lengths to know them
        first = shape_of<ROWS>(a, lane_id());
        double pages = (double)first.tiles * first.pages, tiles = first.tiles;           // sums are exact, being below 2^53
        int longest = first.pages;
#pragma unroll 4
        for (int b0 = 64; b0 < a.seq.count; b0 += 64) {
            const Shape s = shape_of<ROWS>(a, b0 + lane_id());
            pages += (double)s.tiles * s.pages, tiles += s.tiles, longest = max(longest, s.pages);
        }
        if (a.parts) {
            pages = wave_sum(pages) * a.kv_heads;
            const double share = fmin(fmax(pages * (1.0 / DEFAULT_CUS), (double)a.least_share), (double)FULL_SHARE);
            most = uniform((int)fmin(ceil(fmax(pages * (1.0 / PARTS), share)), 0x1p29));
            any = uniform((int)wave_max((uint32_t)longest)) > 2 * most;
        }
        if (any) {
            tiles = (double)first.tiles * cuts(first);
            for (int b0 = 64; b0 < a.seq.count; b0 += 64) {
                const Shape s = shape_of<ROWS>(a, b0 + lane_id());
                tiles += (double)s.tiles * cuts(s);
            }
        }
        if (any || a.seq.cu) items = uniform((int)fmin(wave_sum(tiles) * a.kv_heads, (double)a.most_items));
    }
    __device__ Shape shape(int b) const { return b < 64 ? first : shape_of<ROWS>(a, b); }      // of sequence b, a lane's own in its group of 64
    __device__ Shape at(int b) const                                                           // of any, for all lanes
    {
        if (b >= 64) return shape_of<ROWS>(a, b);
        return {__builtin_amdgcn_readlane(first.tiles, b), __builtin_amdgcn_readlane(first.pages, b)};
    }
    __device__ int cuts(const Shape &s) const { return s.pages > 2 * most ? (s.pages + most - 1) / most : 1; }
};

struct Unit {
    int sequence, head, tile, part, parts, slot;      // sequence -1: there is none; slot: where the part's results go
};
// Item `item` of the list: first the parts of units that are cut, then whole units
template <int ROWS>
__device__ inline Unit find_unit(const DecodeArgs &a, const Shares<ROWS> &shares, int item)
{
    if (!shares.any && !a.seq.cu) {              // as many units of every sequence
        const int tiles = (a.group + ROWS - 1) / ROWS, unit = item % (tiles * a.kv_heads);
        return {item / (tiles * a.kv_heads), unit % a.kv_heads, unit / a.kv_heads, 0, 1, item};
    }
    Found f = {-1, item};
    if (shares.any)
        f = find_sequence(a.seq.count, item, [&](int b) {
            const Shape s = shares.shape(b);
            const int n = shares.cuts(s);
            return n > 1 ? n * s.tiles * a.kv_heads : 0;
        });
    if (f.sequence < 0)
        f = find_sequence(a.seq.count, f.place, [&](int b) {
            const Shape s = shares.shape(b);
            return shares.cuts(s) > 1 ? 0 : s.tiles * a.kv_heads;
        });
    if (f.sequence < 0) return {-1, 0, 0, 0, 1, item};
    const int b = uniform(f.sequence), place = uniform(f.place);
    const int parts = uniform(shares.cuts(shares.at(b))), unit = place / parts;
    return {b, unit % a.kv_heads, unit / a.kv_heads, place % parts, parts, item};
}

__device__ inline uint32_t widen(uint32_t codes, float scale, bool high)
{
    return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes, scale, true)
                                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes, scale, false));
}
// eight codes to a fragment
__device__ inline v8bf fragment(uint32_t a, uint32_t b, float scale)
{
    return __builtin_bit_cast(v8bf, v4u{widen(a, scale, false), widen(a, scale, true), widen(b, scale, false), widen(b, scale, true)});
}

// bytes of a word that are e4m3's NaN, as 0xff each
__device__ inline uint32_t nan_bytes(uint32_t w)
{
    const uint32_t t = (w & 0x7f7f7f7fu) + 0x01010101u;       // bit 7 of a byte: its seven bits are all ones
    return (t >> 7 & 0x01010101u) * 0xffu;
}

// maximum and sum over the four lanes of a column (16 and 32 lanes away)
__device__ inline float column_max(float v)
{
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t w = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
    const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float column_sum(float v)
{
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t w = __float_as_uint(__uint_as_float(a[0]) + __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// maximum over 16 lanes
__device__ inline float row_max(float v)
{
    v = fmaxf(v, __uint_as_float(other_lane<8>(__float_as_uint(v))));
    v = fmaxf(v, __uint_as_float(other_lane<4>(__float_as_uint(v))));
    v = fmaxf(v, __uint_as_float(other_lane<2>(__float_as_uint(v))));
    return fmaxf(v, __uint_as_float(other_lane<1>(__float_as_uint(v))));
}

constexpr float NONE = -__builtin_inff();

template <int D, int RT>
__global__ __launch_bounds__(64 * waves_of(RT), 2) void cached_attention_kernel(const int32_t *lengths, const int32_t *table_at, const int32_t *cu,
                                                                                const uint16_t *q_at, int64_t q_token, int64_t q_head, int32_t kv_heads,
                                                                                int32_t group, const DecodeArgs rest)
{
    // what a workgroup needs first comes with the dispatch
    DecodeArgs a = rest;
    a.seq.lengths = lengths, a.seq.table = table_at, a.seq.cu = cu, a.q = {q_at, q_token, q_head}, a.kv_heads = kv_heads, a.group = group;
    constexpr int ROWS = 16 * RT, KB = D / 64, DG = D / 16, PITCH = D + 4, WAVES = waves_of(RT);
    __shared__ __attribute__((aligned(16))) float sums[WAVES][ROWS][PITCH];
    __shared__ float stats[WAVES][ROWS][2];
    // The grid is for the most parts there can be, up to MAX_GRID; how many there are, and which, is known here only.
    const Shares<ROWS> shares(a);
    for (int item = blockIdx.x; item < shares.items; item += gridDim.x) {
        const Unit u = find_unit<ROWS>(a, shares, item);
        if (u.sequence < 0) return;
        if (item != (int)blockIdx.x) __syncthreads();             // LDS is free again
        int thread = threadIdx.x;
        asm volatile("" : "+v"(thread));             // what follows from it is not kept from part to part: there are no registers for that
        const int lane = thread & 63, wave = uniform(thread >> 6), col = lane & 15, g = lane >> 4;
        const Span span = new_tokens(a.seq, u.sequence);
        const int begin = uniform(span.begin), n = uniform(span.n), length = uniform(length_of(a.seq, u.sequence));
        const int pages = (int)min((int64_t)(length + PAGE - 1) / PAGE, a.seq.table_width);
        const int rows = n * a.group, row0 = u.tile * ROWS;

        // the rows' queries, and how many keys each sees
        // (32 rows of 128 values leave no registers for them: every page reads them from LDS again)
        constexpr bool IN_LDS = RT == 2 && D == 128;
        __shared__ __attribute__((aligned(16))) v8bf shared_q[IN_LDS ? RT * KB * 2 : 1][64];
        v8bf q[RT][KB][2];
        int limit[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int row = row0 + 16 * t + col, token = min(row, rows - 1) / a.group, h = min(row, rows - 1) % a.group;
            limit[t] = row < rows ? max(length - n + 1 + token, 0) : 0;
            const uint16_t *const from = a.q.p + (int64_t)(begin + token) * a.q.token + (int64_t)(u.head * a.group + h) * a.q.head + g * 16;
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int s = 0; s < 2; ++s) q[t][k][s] = __builtin_bit_cast(v8bf, *(const v4u *)(from + k * 64 + s * 8));
        }
        if (IN_LDS) {
            if (wave == 0)
#pragma unroll
                for (int i = 0; i < RT * KB * 2; ++i) shared_q[i][lane] = q[i / (KB * 2)][i / 2 % KB][i % 2];
            __syncthreads();
        }
        const int first_token = row0 / a.group, last_token = (min(row0 + ROWS, rows) - 1) / a.group;
        // keys below it need no mask (of a tile that is not full none do: rows that are not there see nothing, so its pages all take the masked way)
        const int all_see = row0 + ROWS <= rows ? max(length - n + 1 + first_token, 0) : 0;
        const int some_see = max(length - n + 1 + last_token, 0);                                // keys from it on nobody sees

        // this part's pages that anybody sees, this wave's among them
        const int per = (pages + u.parts - 1) / u.parts, from = u.part * per;
        const int to = min(min(from + per, pages), (some_see + PAGE - 1) / PAGE);
        const int mine = max((to - from - wave + WAVES - 1) / WAVES, 0);
        const int32_t *const table = a.seq.table + (int64_t)u.sequence * a.seq.table_width;

        v4f o[RT][DG];
        float m[RT], l[RT];                          // maxima so far, this lane's share of the sums
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            m[t] = NONE, l[t] = 0.0f;
#pragma unroll
            for (int d = 0; d < DG; ++d) o[t][d] = v4f{0, 0, 0, 0};
        }
        const int k_lane = (16 * (col >> 2) + (col & 3)) * 64 + g * 16, v_lane = g * (16 * D) + col * 16;

        // up to 64 of the wave's pages at a time: a lane looks one up (the first of them while the length is on its way)
        const auto look_up = [&](int i0) { return table[min((int64_t)(from + wave + (i0 + lane) * WAVES), a.seq.table_width - 1)]; };
        int id = look_up(0);
        for (int i0 = 0; i0 < mine; i0 += 64) {
            if (i0) id = look_up(i0);
            // A number outside the pool is no page: its tokens are not seen.  Page 0's codes are loaded in its place and become NONE and zeros; their scale is 1
            // and not page 0's, which may never have been written: zero widened by a scale of NaN is NaN.
            if (i0 + lane >= mine || id < 0 || id >= a.cache.pages) id = -1;
            float ks = 1.0f, vs = 1.0f;
            if (id >= 0) {
                const int64_t at = (int64_t)id * a.kv_heads + u.head;
                ks = a.cache.ks[at], vs = a.cache.vs[at];
            }
            const int count = min(mine - i0, 64);
            const auto base_of = [&](int i) { return ((int64_t)max(__builtin_amdgcn_readlane(id, i), 0) * a.kv_heads + u.head) * (PAGE * D); };
            v4u kc[KB][4], vc[DG];
            const auto load_keys = [&](int i) {
                const uint8_t *const p = a.cache.k + base_of(i);
#pragma unroll
                for (int k = 0; k < KB; ++k)
#pragma unroll
                    for (int b = 0; b < 4; ++b) kc[k][b] = *(const v4u *)(p + k_lane + k * (PAGE * 64) + b * 256);
            };
            const auto load_values = [&](int i) {
                const uint8_t *const p = a.cache.v + base_of(i);
#pragma unroll
                for (int d = 0; d < DG; ++d) vc[d] = *(const v4u *)(p + v_lane + d * 256);
            };
            load_keys(0);
            load_values(0);
            for (int i = 0; i < count; ++i) {
                const bool more = i + 1 < count;
                const bool there = __builtin_amdgcn_readlane(id, i) >= 0;
                const float key_scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), i));
                const float value_scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), i));
                const int position = (from + wave + (i0 + i) * WAVES) * PAGE;
                v4f s[RT][4];
                if (IN_LDS) {
                    asm volatile("" ::: "memory");
#pragma unroll
                    for (int i = 0; i < RT * KB * 2; ++i) q[i / (KB * 2)][i / 2 % KB][i % 2] = shared_q[i][lane];
                }
#pragma unroll
                for (int b = 0; b < 4; ++b) {
#pragma unroll
                    for (int t = 0; t < RT; ++t) s[t][b] = v4f{0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < KB; ++k)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const v8bf f = fragment(kc[k][b][2 * h], kc[k][b][2 * h + 1], key_scale);
#pragma unroll
                            for (int t = 0; t < RT; ++t) s[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q[t][k][h], s[t][b], 0, 0, 0);
                        }
                }
                const bool masked = !there || position + PAGE > all_see;
                if (masked) {
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        const int seen = there ? limit[t] - position - 16 * g : 0;         // of the lane's 16 tokens
#pragma unroll
                        for (int b = 0; b < 4; ++b)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[t][b][e] = 4 * b + e < seen ? s[t][b][e] : NONE;
                    }
                    // what nobody sees may hold anything, and 0 times NaN is NaN
                    const int seen = there ? some_see - position - 16 * g : 0;
                    const v4u keep = {seen >= 4 ? ~0u : seen <= 0 ? 0u : (1u << 8 * seen) - 1u, seen >= 8 ? ~0u : seen <= 4 ? 0u : (1u << 8 * (seen - 4)) - 1u,
                                      seen >= 12 ? ~0u : seen <= 8 ? 0u : (1u << 8 * (seen - 8)) - 1u, seen >= 16 ? ~0u : seen <= 12 ? 0u : (1u << 8 * (seen - 12)) - 1u};
#pragma unroll
                    for (int d = 0; d < DG; ++d) vc[d] &= keep;
                    // Nor may a NaN that some rows see reach the others: it is taken out, and the rows that see it are found by a product of indicators.
                    uint32_t bad = 0;
#pragma unroll
                    for (int d = 0; d < DG; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) bad |= nan_bytes(vc[d][e]);
                    if (__any(bad != 0)) {
#pragma unroll
                        for (int d = 0; d < DG; ++d) {
                            v4u hit;
#pragma unroll
                            for (int e = 0; e < 4; ++e) hit[e] = nan_bytes(vc[d][e]), vc[d][e] &= ~hit[e], hit[e] &= 0x38383838u;      // 1.0
#pragma unroll
                            for (int t = 0; t < RT; ++t) {
                                const int rows_see = there ? limit[t] - position - 16 * g : 0;
                                v4f times = {0, 0, 0, 0};
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    v4u see;
#pragma unroll
                                    for (int e = 0; e < 4; ++e) see[e] = (8 * h + 2 * e < rows_see ? 0x3f80u : 0u) | (8 * h + 2 * e + 1 < rows_see ? 0x3f800000u : 0u);
                                    times = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fragment(hit[2 * h], hit[2 * h + 1], 1.0f), __builtin_bit_cast(v8bf, see), times, 0, 0, 0);
                                }
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (times[e] > 0.0f) o[t][d][e] = __builtin_nanf("");
                            }
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
                if (more) load_keys(i + 1);
                uint32_t p[RT][8];
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    float top = s[t][0][0];
#pragma unroll
                    for (int e = 1; e < 16; ++e) top = fmaxf(top, s[t][e >> 2][e & 3]);
                    top *= a.scale;
                    if (__any(top > m[t] + 8.0f)) {
                        const float grown = fmaxf(m[t], column_max(top));
                        const float by = m[t] == NONE ? 0.0f : __builtin_amdgcn_exp2f(m[t] - grown);
                        m[t] = grown;
                        l[t] *= by;
#pragma unroll
                        for (int d = 0; d < DG; ++d) o[t][d] *= by;
                    }
                    const float base = m[t] == NONE ? 0.0f : m[t];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e >> 1][2 * (e & 1)], a.scale, -base));
                        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e >> 1][2 * (e & 1) + 1], a.scale, -base));
                        l[t] += x + y;
                        p[t][e] = pack_bf16(x, y);
                    }
                }
#pragma unroll
                for (int d = 0; d < DG; ++d) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const v8bf f = fragment(vc[d][2 * h], vc[d][2 * h + 1], value_scale);
#pragma unroll
                        for (int t = 0; t < RT; ++t)
                            o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, __builtin_bit_cast(v8bf, v4u{p[t][4 * h], p[t][4 * h + 1], p[t][4 * h + 2], p[t][4 * h + 3]}), o[t][d], 0, 0, 0);
                    }
                }
                if (more) load_values(i + 1);
            }
        }

        // the waves' results, brought to one maximum
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const float sum = column_sum(l[t]);
            if (g == 0) stats[wave][16 * t + col][0] = m[t], stats[wave][16 * t + col][1] = sum;
#pragma unroll
            for (int d = 0; d < DG; ++d) *(v4f *)&sums[wave][16 * t + col][16 * d + 4 * g] = o[t][d];
        }
        __syncthreads();
        constexpr int PER_ROW = D / 8;
        for (int at = thread; at < ROWS * PER_ROW; at += 64 * WAVES) {
            const int row = at / PER_ROW, d0 = at % PER_ROW * 8;
            if (row0 + row >= rows) continue;
            float top = NONE, weight = 0.0f;
            for (int w = 0; w < WAVES; ++w) top = fmaxf(top, stats[w][row][0]);
            v4f x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
            for (int w = 0; w < WAVES; ++w) {
                // a wave that has seen nothing: zero sums, or NaN where a score was one
                const float mw = stats[w][row][0], by = mw == NONE ? 1.0f : __builtin_amdgcn_exp2f(mw - top);
                weight += by * stats[w][row][1];
                x += by * *(const v4f *)&sums[w][row][d0], y += by * *(const v4f *)&sums[w][row][d0 + 4];
            }
            if (u.parts > 1) {
                float *const to_sums = a.parts + ((int64_t)u.slot * ROWS + row) * D + d0;
                *(v4f *)to_sums = x, *(v4f *)(to_sums + 4) = y;
                if (d0 == 0) {
                    float *const to_stats = a.parts + (int64_t)2 * PARTS * ROWS * D + ((int64_t)u.slot * ROWS + row) * 2;
                    to_stats[0] = top, to_stats[1] = weight;
                }
            } else {
                const float r = weight == 0.0f ? 0.0f : 1.0f / weight;          // a row that sees nothing: zeros
                const int token = begin + (row0 + row) / a.group, h = u.head * a.group + (row0 + row) % a.group;
                *(v4u *)(a.out + ((int64_t)token * a.heads + h) * D + d0) =
                    v4u{pack_bf16(x[0] * r, x[1] * r), pack_bf16(x[2] * r, x[3] * r), pack_bf16(y[0] * r, y[1] * r), pack_bf16(y[2] * r, y[3] * r)};
            }
        }
        if (D == 128 && RT == 2) return;             // no registers to go on with: its grid has a workgroup for every part
    }
}

// Joins the parts of a unit that was cut, a row to a wave, or to the waves of a workgroup, which then take every eighth part.  blockIdx.y: the unit.
template <int D, int RT>
__global__ __launch_bounds__(64 * JOIN_WAVES) void join_parts_kernel(const DecodeArgs a, int waves_a_row)
{
    constexpr int ROWS = 16 * RT, E = D / 64;
    __shared__ float sums[JOIN_WAVES][D], stats[JOIN_WAVES][2];
    const Shares<ROWS> shares(a);
    if (!shares.any) return;
    const auto cut = [&](const Shape &s) { return shares.cuts(s) > 1; };
    for (int y = blockIdx.y;; y += gridDim.y) {
        const Found f = find_sequence(a.seq.count, y, [&](int b) {
            const Shape s = shares.shape(b);
            return cut(s) ? s.tiles * a.kv_heads : 0;
        });
        if (f.sequence < 0) return;
        if (y != (int)blockIdx.y) __syncthreads();                // LDS is free again
        const int b = uniform(f.sequence), unit = uniform(f.place), tile = unit / a.kv_heads, head = unit % a.kv_heads;
        const int parts = uniform(shares.cuts(shares.at(b)));
        const Span span = new_tokens(a.seq, b);
        const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
        const int row = waves_a_row == 1 ? blockIdx.x * JOIN_WAVES + wave : blockIdx.x, first = waves_a_row == 1 ? 0 : wave;
        const int at = tile * ROWS + row;
        const bool live = row < ROWS && at < uniform(span.n) * a.group;
        if (!live && waves_a_row == 1) continue;
        // parts of the cut units before this one's
        double before = 0.0;
        for (int b0 = 0; b0 < b; b0 += 64) {
            const Shape s = shares.shape(b0 + lane);
            before += b0 + lane < b && cut(s) ? shares.cuts(s) * s.tiles * a.kv_heads : 0;
        }
        const int slot = uniform((int)wave_sum(before)) + unit * parts;
        const float *const from = a.parts + ((int64_t)slot * ROWS + min(row, ROWS - 1)) * D + lane * E;
        const float *const stat = a.parts + (int64_t)2 * PARTS * ROWS * D + ((int64_t)slot * ROWS + min(row, ROWS - 1)) * 2;
        float x[E] = {}, top = NONE, weight = 0.0f;
        // 64 parts at a time: a lane has the maximum and the weight of one; then their sums, whose loads wait for nothing
        for (int p0 = first; live && p0 < parts; p0 += 64 * waves_a_row) {
            const int p = p0 + lane * waves_a_row;
            const float2 own = p < parts ? *(const float2 *)(stat + (int64_t)p * ROWS * 2) : float2{NONE, 0.0f};
            const float grown = fmaxf(top, column_max(row_max(own.x)));
            const float old = top == NONE ? 1.0f : __builtin_amdgcn_exp2f(top - grown), by = own.x == NONE ? 1.0f : __builtin_amdgcn_exp2f(own.x - grown);
            weight = weight * old + (float)wave_sum((double)(own.y * by));
            top = grown;
            const int n = min((parts - p0 + waves_a_row - 1) / waves_a_row, 64);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] *= old;
            for (int i0 = 0; i0 < n; i0 += 8)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int part = min(i0 + i, n - 1);
                    const float w = i0 + i < n ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(by), part)) : 0.0f;
                    const float *const y = from + (int64_t)(p0 + part * waves_a_row) * ROWS * D;
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] += w * y[e];
                }
        }
        if (waves_a_row > 1) {
#pragma unroll
            for (int e = 0; e < E; ++e) sums[wave][lane * E + e] = x[e];
            if (lane == 0) stats[wave][0] = top, stats[wave][1] = weight;
            __syncthreads();
            if (wave > 0 || !live) continue;
            for (int i = 0; i < JOIN_WAVES; ++i) top = fmaxf(top, stats[i][0]);
            weight = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = 0.0f;
            for (int i = 0; i < JOIN_WAVES; ++i) {
                const float by = stats[i][0] == NONE ? 1.0f : __builtin_amdgcn_exp2f(stats[i][0] - top);
                weight += by * stats[i][1];
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] += by * sums[i][lane * E + e];
            }
        }
        const int token = uniform(span.begin) + at / a.group, h = head * a.group + at % a.group;
        uint16_t *const to = a.out + ((int64_t)token * a.heads + h) * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) to[e] = bf16_rne(weight == 0.0f ? 0.0f : x[e] / weight);
    }
}

// Rows of a tile: 16, or 32 where the sequences have more on average
static int row_tiles(int64_t tokens, int64_t sequences, int group) { return tokens * group > 16 * sequences ? 2 : 1; }

// What the host knows of a launch: units (row tiles of every sequence and kv head) and their pages, as many as there can be
static int64_t most_units(int64_t tokens, int64_t sequences, int group, int kv_heads, int rows)
{
    const int64_t tiles = tokens * group / rows + sequences;        // of n rows: n / rows + 1 at most
    return (tiles < tokens * group ? tiles : tokens * group) * kv_heads;
}
static int64_t most_cut(int64_t units, int64_t table_width)         // parts of cut units
{
    const int least = least_share(units);
    if (table_width <= 2 * least) return 0;
    const int64_t by_width = units * ((table_width + least - 1) / least);
    return by_width < 2 * PARTS ? by_width : 2 * PARTS;
}

int64_t cached_attention_scratch_bytes(int64_t tokens, int64_t sequences, int heads, int kv_heads, int head_dim, int64_t table_width)
{
    const int group = heads / kv_heads, rows = 16 * row_tiles(tokens, sequences, group);
    return most_cut(most_units(tokens, sequences, group, kv_heads, rows), table_width) ? (int64_t)2 * PARTS * rows * (head_dim + 2) * 4 : 0;
}

hipError_t launch_cached_attention(Heads q, const Sequences &s, int heads, int kv_heads, int head_dim, float scale, const Cache &cache, uint16_t *out,
                                   uint8_t *scratch, int64_t scratch_bytes, hipStream_t stream)
{
    const int group = heads / kv_heads, tiles = row_tiles(s.tokens, s.count, group), rows = 16 * tiles;
    const int64_t units = most_units(s.tokens, s.count, group, kv_heads, rows);
    const int64_t need = cached_attention_scratch_bytes(s.tokens, s.count, heads, kv_heads, head_dim, s.table_width);
    const bool cut = need > 0 && scratch && scratch_bytes >= need;
    DecodeArgs a = {q, s, cache, out, cut ? (float *)scratch : nullptr, heads, kv_heads, group, scale * 1.44269504088896341f, 0, least_share(units)};
    const int64_t items = units + (cut ? most_cut(units, s.table_width) : 0), grid = items < MAX_GRID || (head_dim == 128 && tiles == 2) ? items : MAX_GRID;
    if (items > 1 << 23) return hipErrorInvalidConfiguration;      // before the device is asked for anything; n * group fits in 32 bits then
    const DeviceInfo *info;
    hipError_t e = device_info(&info);
    if (e != hipSuccess) return e;
    a.most_items = (int)items;
    const dim3 threads(64 * waves_of(tiles)), blocks((unsigned)grid);
    const auto kernel = head_dim == 128 ? tiles == 1 ? cached_attention_kernel<128, 1> : cached_attention_kernel<128, 2>
                                        : tiles == 1 ? cached_attention_kernel<64, 1> : cached_attention_kernel<64, 2>;
    kernel<<<blocks, threads, 0, stream>>>(s.lengths, s.table, s.cu, q.p, q.token, q.head, kv_heads, group, a);
    if (cut) {
        const int most = units < JOINED ? (int)units : JOINED, used = s.cu || group > rows ? rows : group;
        // with few rows several waves to each: a unit may have many parts then (4 tokens behind 131072, 64 parts: 4.4 us)
        const int waves_a_row = (int64_t)most * used <= 512 ? JOIN_WAVES : 1;
        const dim3 joins((unsigned)(waves_a_row == 1 ? (used + JOIN_WAVES - 1) / JOIN_WAVES : used), (unsigned)most);
        const auto join = head_dim == 128 ? tiles == 1 ? join_parts_kernel<128, 1> : join_parts_kernel<128, 2>
                                          : tiles == 1 ? join_parts_kernel<64, 1> : join_parts_kernel<64, 2>;
        join<<<joins, dim3(64 * JOIN_WAVES), 0, stream>>>(a, waves_a_row);
    }
    return hipGetLastError();
}

}  // namespace fptq
