// Appending to the paged 8-bit cache, with the position rotation on the way.
//
// A page-head (64 tokens of one kv head) holds e4m3 codes c and one scale s, a power of two: x ~ c s, s the smallest with max |x| <= 448 s.  A
// power of two, because then older codes move to a larger scale by an exponent, c' = rne(c 2^-n), and the attention's widening to bf16 takes
// the scale for nothing and exactly.  Keys are rotated in fp32 (every product and sum rounded by itself, no contraction) and rounded once, to the code.
//
// A launch for everything: a workgroup for the keys or the values of a page-head, whose scale needs all of the page's new tokens, and waves for the queries of a
// token, which keep its angles over the heads.  Values are read a row a wave and written transposed, 16 tokens a lane, from registers.
// Measured (the kernel; a call among others): a prompt of 4096 tokens, 32 heads over 8 of 128, 103 MB read and written: 19.6 us, 5.2 TB/s; 19.5 to 23.  A token 4.1 us;
// 5.8 to 6.0: a chain of latencies (length, angles, page, its scale and codes) of which the rows' own is taken out by reading them first.
#include "fptq_attention.h"

namespace fptq {

typedef float v2f __attribute__((ext_vector_type(2)));

// bits of the smallest power of two s with largest <= 448 s, 2^-100 at least: 448 is 1.75 * 2^8, so the mantissa's carry past 1.75 raises the exponent
__device__ inline uint32_t scale_bits(uint32_t largest) { return (uint32_t)max((int)((largest + 0x1fffffu) >> 23) - 8, 27) << 23; }
// bits of 1 / s of a power of two between 2^-126 and 2^126
__device__ inline float reciprocal_of(uint32_t scale) { return __uint_as_float((254u << 23) - scale); }

// What a value in units of the scale is held to where the scale is the largest there is: from 248 on the nearest code would be 256, which is worth
// 2^128 and infinite in the bf16 that the attention widens it to.  240 is within half a step's 2^-4 of all that a float can be there; what is not finite stays so.
constexpr float LARGEST_SCALE = 0x1p120f;
__device__ inline float below_infinity(float y) { return fabsf(y) < 256.0f ? fminf(fmaxf(y, -240.0f), 240.0f) : y; }

// |x| as it counts for the scale: what is not finite does not, and is stored as NaN
__device__ inline uint32_t magnitude(float x)
{
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

// four values in units of the scale, rounded to nearest even; the conversion makes NaN of what is beyond 464, infinities and NaN
__device__ inline uint32_t codes(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// four older codes in the unit of a larger scale
__device__ inline uint32_t rescaled(uint32_t w, float ratio)
{
    const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return codes(lo.x * ratio, lo.y * ratio, hi.x * ratio, hi.y * ratio);
}

// bytes of a word of four tokens t0 .. t0 + 3 that lie in [from, to)
__device__ inline uint32_t bytes_between(int t0, int from, int to)
{
    const int a = min(max(from - t0, 0), 4), b = min(max(to - t0, 0), 4);
    const uint32_t below_b = b == 4 ? 0xffffffffu : (1u << (8 * b)) - 1u, below_a = a == 4 ? 0xffffffffu : (1u << (8 * a)) - 1u;
    return below_b & ~below_a;
}

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The rotation of a row is done 16 values a thread: two runs of eight, whose first values are lo and hi.  Half layout: values i and i + R / 2 of the R
// rotated ones are a pair.  Interleaved: 2 i and 2 i + 1.  Both take frequencies 8 u .. 8 u + 7 of the table's row.
struct Runs {
    int lo, hi;
    bool rotated;
};
__device__ inline Runs runs_of(int u, int rope_dims, bool interleaved)
{
    const bool rotated = 16 * u < rope_dims;
    const bool half = rotated && !interleaved;
    return {half ? 8 * u : 16 * u, half ? rope_dims / 2 + 8 * u : 16 * u + 8, rotated};
}

struct Angles {
    float c[8], s[8];
};
// of position `position`; outside the table: NaN, so that the mistake is seen
__device__ inline Angles angles_of(const float *rope, int64_t positions, int rope_dims, int position, int u, bool rotated)
{
    Angles a;
    const bool known = position >= 0 && position < positions;
#pragma unroll
    for (int e = 0; e < 8; ++e) a.c[e] = rotated ? __uint_as_float(0x7fc00000u) : 1.0f, a.s[e] = 0.0f;
    if (rotated && known) {
        const float4 *const p = (const float4 *)(rope + (int64_t)position * rope_dims + 8 * u);
        const float4 *const q = (const float4 *)(rope + (int64_t)position * rope_dims + rope_dims / 2 + 8 * u);
        const float4 c0 = p[0], c1 = p[1], s0 = q[0], s1 = q[1];
        a = {{c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w}};
    }
    return a;
}

// x[0 .. 7], x[8 .. 15]: the two runs
template <bool INTERLEAVED>
__device__ inline void rotate(float (&x)[16], const v4u lo, const v4u hi, const Angles &t, bool rotated)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = bf16_lo(lo[e]), x[2 * e + 1] = bf16_hi(lo[e]);
        x[8 + 2 * e] = bf16_lo(hi[e]), x[8 + 2 * e + 1] = bf16_hi(hi[e]);
    }
    if (!rotated) return;
    if (INTERLEAVED) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = x[2 * e], b = x[2 * e + 1];
            x[2 * e] = a * t.c[e] - b * t.s[e], x[2 * e + 1] = b * t.c[e] + a * t.s[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = x[e], b = x[8 + e];
            x[e] = a * t.c[e] - b * t.s[e], x[8 + e] = b * t.c[e] + a * t.s[e];
        }
    }
}

__device__ inline v4u packed(const float *x) { return v4u{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])}; }

struct AppendArgs {
    Heads q, k, v;
    Sequences seq;
    Cache cache;
    const float *rope;
    int64_t positions;
    uint16_t *q_out, *k_out;
    int heads, kv_heads, rope_dims;
    int page_slots, query_parts;         // pages that the new tokens can touch; waves a token's query heads are spread over
};

// A sequence's new tokens and the position of the first of them (negative for a length that does not count them)
struct Place {
    int sequence, begin, n, at;
};
__device__ inline Place place_of(const Sequences &s, int b)
{
    const Span span = new_tokens(s, b);
    return {b, span.begin, span.n, length_of(s, b) - span.n};
}
// The first sequence for which `is` holds, all lanes with one each; 64 a step.  sequence -1: none.
template <class Is>
__device__ inline Place first_of(const Sequences &s, Is is)
{
    const int lane = lane_id();
    for (int b0 = 0; b0 < s.count; b0 += 64) {
        const Place own = b0 + lane < s.count ? place_of(s, b0 + lane) : Place{-1, 0, 0, 0};
        const uint64_t hit = __ballot(is(own));
        if (hit) {
            const int at = __builtin_ctzll(hit);
            return {b0 + at, __builtin_amdgcn_readlane(own.begin, at), __builtin_amdgcn_readlane(own.n, at), __builtin_amdgcn_readlane(own.at, at)};
        }
    }
    return {-1, 0, 0, 0};
}

// The new tokens of one page: rows first .. last - 1 of it, tokens from `token` on
struct PageRows {
    int first, last, token, position;    // position: of row 0
    const int32_t *entry;                // of the table, NULL if it has none
};
__device__ inline bool page_rows(const Sequences &s, int slot, PageRows &r)
{
    Place p;
    int before = 0;                      // pages that sequences before this one touch
    if (s.cu) {
        int all = 0;
        p = first_of(s, [&](const Place &i) {
            const int own = i.n > 0 ? ((i.at + i.n - 1) >> 6) - (i.at >> 6) + 1 : 0, upto = all + wave_prefix(own);
            all = __builtin_amdgcn_readlane(upto, 63);
            const uint64_t hit = __ballot(slot < upto);
            if (hit) before = __builtin_amdgcn_readlane(upto - own, __builtin_ctzll(hit));
            return slot < upto;
        });
    } else if (slot < s.count) {
        p = place_of(s, slot);
        p.at = uniform(p.at);
    } else {
        return false;
    }
    if (p.sequence < 0) return false;
    const int page = (p.at >> 6) + slot * (s.cu ? 1 : 0) - before;
    r.position = page * PAGE;
    r.first = max(p.at - r.position, 0), r.last = min(p.at + p.n - r.position, PAGE);
    r.token = p.begin + r.position + r.first - p.at;
    r.entry = page >= 0 && page < s.table_width ? s.table + (int64_t)p.sequence * s.table_width + page : nullptr;
    return true;
}
// its number, -1 if the table names none of the cache
__device__ inline int64_t page_number(const AppendArgs &a, const PageRows &r)
{
    const int page = r.entry ? uniform(*r.entry) : -1;
    return page >= 0 && page < a.cache.pages ? page : -1;
}

// the largest magnitude over a workgroup of four waves
__device__ inline uint32_t workgroup_max(uint32_t v, uint32_t *lds)
{
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return max(max(lds[0], lds[1]), max(lds[2], lds[3]));
}

// A page-head of keys.  Its codes lie as [D / 64][64 tokens][64 values].
template <int D, bool INTERLEAVED>
__device__ inline void append_keys(const AppendArgs &a, const PageRows &r, int j, uint32_t *lds)
{
    constexpr int U = D / 16, ROWS = 256 / U, PASSES = PAGE / ROWS;
    const int u = threadIdx.x % U, row0 = threadIdx.x / U;
    const Runs run = runs_of(u, a.rope_dims, INTERLEAVED);
    // the rows first, which need no page
    v4u lo[PASSES], hi[PASSES];
    Angles angles[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int row = min(max(row0 + p * ROWS, r.first), r.last - 1);
        const uint16_t *const from = a.k.p + (int64_t)(r.token + row - r.first) * a.k.token + j * a.k.head;
        lo[p] = *(const v4u *)(from + run.lo), hi[p] = *(const v4u *)(from + run.hi);
        angles[p] = angles_of(a.rope, a.positions, a.rope_dims, r.position + row, u, run.rotated);
    }
    const int64_t page = page_number(a, r);
    uint8_t *const to = a.cache.k + (page * a.kv_heads + j) * (PAGE * D);
    float *const scale_at = a.cache.ks + page * a.kv_heads + j;
    constexpr int GRANULES = D / 64 * PAGE * 4 / 256;
    v4u old[GRANULES];
    float old_scale = 0.0f;
    const bool older = page >= 0 && r.first > 0;
    if (older) {
        old_scale = *scale_at;
#pragma unroll
        for (int i = 0; i < GRANULES; ++i) old[i] = *(const v4u *)(to + (i * 256 + threadIdx.x) * 16);
    }
    float x[PASSES][16];
    uint32_t largest = 0;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int row = row0 + p * ROWS;
        rotate<INTERLEAVED>(x[p], lo[p], hi[p], angles[p], run.rotated);
        if (row >= r.first && row < r.last) {
#pragma unroll
            for (int e = 0; e < 16; ++e) largest = max(largest, magnitude(x[p][e]));
            if (a.k_out) {
                uint16_t *const out = a.k_out + ((int64_t)(r.token + row - r.first) * a.kv_heads + j) * D;
                *(v4u *)(out + run.lo) = packed(x[p]), *(v4u *)(out + run.hi) = packed(x[p] + 8);
            }
        }
    }
    largest = workgroup_max(largest, lds);
    if (page < 0) return;
    const float scale = fmaxf(__uint_as_float(scale_bits(largest)), old_scale), unit = reciprocal_of(__float_as_uint(scale));
    if (threadIdx.x == 0) *scale_at = scale;
    if (older && scale > old_scale) {
#pragma unroll
        for (int i = 0; i < GRANULES; ++i) {
            const int granule = i * 256 + threadIdx.x;
            if (granule / 4 % PAGE < r.first) {
                v4u w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = rescaled(old[i][e], old_scale * unit);
                *(v4u *)(to + granule * 16) = w;
            }
        }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int row = row0 + p * ROWS;
        if (row >= r.first && row < r.last) {
            float *const y = x[p];
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] *= unit;
            if (scale == LARGEST_SCALE)
#pragma unroll
                for (int e = 0; e < 16; ++e) y[e] = below_infinity(y[e]);
            uint2 lo = {codes(y[0], y[1], y[2], y[3]), codes(y[4], y[5], y[6], y[7])};
            uint2 hi = {codes(y[8], y[9], y[10], y[11]), codes(y[12], y[13], y[14], y[15])};
            *(uint2 *)(to + run.lo / 64 * (PAGE * 64) + row * 64 + run.lo % 64) = lo;
            *(uint2 *)(to + run.hi / 64 * (PAGE * 64) + row * 64 + run.hi % 64) = hi;
        }
    }
}

// A page-head of values.  Its codes lie as [4][D][16 tokens]: a wave takes 16 tokens, a lane the D / 64 values of each, and writes them as whole runs.
template <int D>
__device__ inline void append_values(const AppendArgs &a, const PageRows &r, int j, uint32_t *lds)
{
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63, t0 = threadIdx.x >> 6 << 4, d0 = lane * E;
    const int first = min(max(r.first - t0, 0), 16), last = min(max(r.last - t0, 0), 16);
    const bool whole = first == 0 && last == 16;
    uint32_t w[16];                      // the rows first, which need no page
#pragma unroll
    for (int t = 0; t < 16; ++t) {
        w[t] = 0;
        if (t >= first && t < last) {
            const uint16_t *const from = a.v.p + (int64_t)(r.token + t0 + t - r.first) * a.v.token + j * a.v.head + d0;
            w[t] = E == 2 ? *(const uint32_t *)from : *from;
        }
    }
    const int64_t page = page_number(a, r);
    uint8_t *const to = a.cache.v + (page * a.kv_heads + j) * (PAGE * D) + t0 * D + d0 * 16;
    float *const scale_at = a.cache.vs + page * a.kv_heads + j;
    v4u old[E];
    float old_scale = 0.0f;
    if (page >= 0) {
        if (r.first > 0) old_scale = *scale_at;
        if (!whole) {
#pragma unroll
            for (int e = 0; e < E; ++e) old[e] = *(const v4u *)(to + 16 * e);
        }
    }
    float x[E][16];
    uint32_t largest = 0;
#pragma unroll
    for (int t = 0; t < 16; ++t) {
        x[0][t] = bf16_lo(w[t]);
        if (E == 2) x[E - 1][t] = bf16_hi(w[t]);
#pragma unroll
        for (int e = 0; e < E; ++e) largest = max(largest, magnitude(x[e][t]));
    }
    largest = workgroup_max(largest, lds);
    if (page < 0) return;
    const float scale = fmaxf(__uint_as_float(scale_bits(largest)), old_scale), unit = reciprocal_of(__float_as_uint(scale));
    if (threadIdx.x == 0) *scale_at = scale;
    const bool raised = first > 0 && scale > old_scale;
    if (last <= first && !raised) return;
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
        for (int t = 0; t < 16; ++t) x[e][t] *= unit;
        if (scale == LARGEST_SCALE)
#pragma unroll
            for (int t = 0; t < 16; ++t) x[e][t] = below_infinity(x[e][t]);
        v4u w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = codes(x[e][4 * i], x[e][4 * i + 1], x[e][4 * i + 2], x[e][4 * i + 3]);
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t fresh = bytes_between(4 * i, first, last), before = bytes_between(4 * i, 0, first);
                const uint32_t moved = raised ? rescaled(old[e][i], old_scale * unit) : old[e][i];
                w[i] = (w[i] & fresh) | (moved & before) | (old[e][i] & ~(fresh | before));
            }
        }
        *(v4u *)(to + 16 * e) = w;
    }
}

// Query heads of a token: D / 16 threads a head, the wave's angles kept over its heads.
template <int D, bool INTERLEAVED>
__device__ inline void rotate_queries(const AppendArgs &a, int wave)
{
    constexpr int U = D / 16, HEADS = 64 / U;
    const Sequences &s = a.seq;
    const int token = wave / a.query_parts, part = wave % a.query_parts;
    if (token >= s.tokens) return;
    const Place p = s.cu ? first_of(s, [=](const Place &i) { return token >= i.begin && token < i.begin + i.n; }) : place_of(s, token);
    if (p.sequence < 0) return;                          // of no sequence
    const int position = p.at + token - p.begin;
    const int lane = threadIdx.x & 63, u = lane % U;
    const Runs run = runs_of(u, a.rope_dims, INTERLEAVED);
    const Angles t = angles_of(a.rope, a.positions, a.rope_dims, position, u, run.rotated);
    for (int h = part * HEADS + lane / U; h < a.heads; h += a.query_parts * HEADS) {
        const uint16_t *const from = a.q.p + (int64_t)token * a.q.token + h * a.q.head;
        const v4u lo = *(const v4u *)(from + run.lo), hi = *(const v4u *)(from + run.hi);
        float x[16];
        rotate<INTERLEAVED>(x, lo, hi, t, run.rotated);
        uint16_t *const out = a.q_out + ((int64_t)token * a.heads + h) * D;
        *(v4u *)(out + run.lo) = packed(x), *(v4u *)(out + run.hi) = packed(x + 8);
    }
}

// Workgroups: keys and values of every page and kv head (the pages' scales need all of a page's new tokens), then the queries.
template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendArgs a)
{
    __shared__ uint32_t lds[4];
    const int units = a.page_slots * a.kv_heads * 2, unit = blockIdx.x;
    if (unit >= units) {
        rotate_queries<D, INTERLEAVED>(a, (unit - units) * 4 + uniform((int)threadIdx.x >> 6));
        return;
    }
    const int j = unit % a.kv_heads, slot = unit / a.kv_heads >> 1;
    PageRows r;
    if (!page_rows(a.seq, slot, r)) return;
    if (unit / a.kv_heads & 1) append_values<D>(a, r, j, lds);
    else append_keys<D, INTERLEAVED>(a, r, j, lds);
}

hipError_t launch_cache_append(Heads q, Heads k, Heads v, const Sequences &s, int heads, int kv_heads, int head_dim, const float *rope, int64_t positions,
                               int rope_dims, bool interleaved, const Cache &cache, uint16_t *q_out, uint16_t *k_out, hipStream_t stream)
{
    AppendArgs a = {q, k, v, s, cache, rope, positions, q_out, k_out, heads, kv_heads, rope_dims, 0, 0};
    // a sequence of n new tokens touches at most n / 64 + 2 pages, and no more than n
    a.page_slots = s.cu ? (int)(s.tokens < s.tokens / PAGE + 2 * (int64_t)s.count ? s.tokens : s.tokens / PAGE + 2 * (int64_t)s.count) : s.count;
    const int groups = (heads * (head_dim / 16) + 63) / 64;
    a.query_parts = (int64_t)s.tokens * groups <= 4096 ? groups : 1;
    const int64_t blocks = (int64_t)a.page_slots * kv_heads * 2 + ((int64_t)s.tokens * a.query_parts + 3) / 4;
    if (blocks * 256 >= (int64_t)1 << 32) return hipErrorInvalidConfiguration;      // before the device is asked for anything
    const DeviceInfo *info;
    hipError_t e = device_info(&info);
    if (e != hipSuccess) return e;
    const auto kernel = head_dim == 128 ? interleaved ? cache_append_kernel<128, true> : cache_append_kernel<128, false>
                                        : interleaved ? cache_append_kernel<64, true> : cache_append_kernel<64, false>;
    kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace fptq
