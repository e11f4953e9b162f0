// What the kernels between the QKV and the O projection share: how rows of heads, sequences and the 8-bit cache lie, and how a kernel
// finds its part of a ragged batch.
#pragma once

#include "fptq_common.h"

namespace fptq {

constexpr int PAGE = 64;         // tokens of a page of the cache

// bf16 rows of heads, strides in values
struct Heads {
    const uint16_t *p;
    int64_t token, head;
};

struct Cache {
    uint8_t *k, *v;              // [pages][kv_heads][PAGE * D]
    float *ks, *vs;              // [pages][kv_heads]
    int64_t pages;
};

// The sequences of a call.  cu == NULL: one new token each.  lengths count a sequence's tokens with the new ones.
struct Sequences {
    const int32_t *cu, *lengths, *table;
    int32_t count, tokens;
    int64_t table_width;
};

// Where sequence b's new tokens lie, whatever the array holds: begin and begin + n are within the rows.
struct Span {
    int begin, n;
};
__device__ inline Span new_tokens(const Sequences &s, int b)
{
    if (!s.cu) return {b, 1};
    const int begin = min(max(s.cu[b], 0), s.tokens);
    return {begin, max(min(s.cu[b + 1], s.tokens) - begin, 0)};
}

// A sequence's length, small enough that positions do not overflow
__device__ inline int length_of(const Sequences &s, int b) { return min(max(s.lengths[b], 0), 1 << 30); }

__device__ inline int lane_id() { return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)); }

__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// sums over the lanes up to each one, in row shifts and broadcasts of rows' last lanes (__shfl_up's way through LDS takes six times as long)
__device__ inline int wave_prefix(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);      // row_shr:1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);      // row_bcast:15 to rows 1 and 3, row_bcast:31 to rows 2 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
    return v;
}

// Of a list that holds count(b) items of every sequence b, one sequence after the other: the sequence that item `item` belongs to (uniform over
// the wave) and the item's place among that sequence's, or -1 and the items left over if the list is shorter.  64 sequences a step.
struct Found {
    int sequence, place;
};
template <class Count>
__device__ inline Found find_sequence(int sequences, int item, Count count)
{
    int lane = lane_id();
    asm volatile("" : "+v"(lane));       // no address of it is kept over a caller's loops
    for (int b0 = 0; b0 < sequences; b0 += 64) {
        const int own = b0 + lane < sequences ? count(b0 + lane) : 0, upto = wave_prefix(own);
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (item < all) {
            const int at = __builtin_ctzll(__ballot(item < upto));
            return {b0 + at, item - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(own, at))};
        }
        item -= all;
    }
    return {-1, item};
}

// launchers
hipError_t launch_cache_append(Heads q, Heads k, Heads v, const Sequences &s, int heads, int kv_heads, int head_dim, const float *rope, int64_t positions,
                               int rope_dims, bool interleaved, const Cache &cache, uint16_t *q_out, uint16_t *k_out, hipStream_t stream);
int64_t cached_attention_scratch_bytes(int64_t tokens, int64_t sequences, int heads, int kv_heads, int head_dim, int64_t table_width);
hipError_t launch_cached_attention(Heads q, const Sequences &s, int heads, int kv_heads, int head_dim, float scale, const Cache &cache, uint16_t *out,
                                   uint8_t *scratch, int64_t scratch_bytes, hipStream_t stream);
hipError_t launch_prompt_attention(Heads q, Heads k, Heads v, const Sequences &s, int heads, int kv_heads, int head_dim, float scale, uint16_t *out,
                                   hipStream_t stream);

}  // namespace fptq
