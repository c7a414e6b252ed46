// The quantised cache: geometry of its pages and what its kernels share.
//
// A page holds block_tokens tokens of all KV heads of one layer, head after head; a head's part is a row of granules of
// 16 tokens.  A granule is what a wave reads for one matrix instruction, in the order in which the lanes of that
// instruction hold it, so that the attention loads every code as part of 16 bytes per lane and moves none between lanes.
// Lane = 16 * q + i, q = 0..3, i = 0..15:
//   K codes  the product over channels takes 16 tokens x 32 channels at a time, lane (q, i) holds token i, channels
//            32 g + 8 q ... + 7 of block g = 0..3.  4 bits: [token][q][g] words; 8 bits: [g / 2][token][q][g % 2] pairs of words
//   V codes  the product over tokens takes 16 channels x 32 tokens, lane (q, i) holds tokens 4 q ... 4 q + 3 of two granules,
//            channels 8 i ... + 7 one after the other.  [half][q][i][token % 4] words of 8 channels (4 bits, one half) or
//            of 4 (8 bits, half h: channels 8 i + 4 h ...)
//   K scales [q][group][token % 4], token = 4 q + ...: as the lanes hold the result of the product over channels
//   K zeros  [token][group]: an operand of one more product, with the sums of the query's groups
//   V parameters [q][group][4 scales, 4 zeros]: pairs of tokens, for packed arithmetic
// A word's codes are in the order of the channels, low bits first.  Every piece of a token's row is 2 bytes or more and
// belongs to that token alone: rows are written without reading their neighbours.
#pragma once

#include "kvc_device.h"

namespace kvc {

constexpr int kGranule = 16;                 // tokens
constexpr float kTopF16 = 65504.0f;

struct GranuleMap {
    int v_codes, k_scales, k_zeros, v_params, bytes;       // offsets inside a granule; the K codes come first
};
__host__ __device__ constexpr GranuleMap granule_map(int bits_k, int bits_v, int group)
{
    const int groups = kDim / group;
    GranuleMap m = {};
    m.v_codes = 256 * bits_k;
    m.k_scales = m.v_codes + 256 * bits_v;
    m.k_zeros = m.k_scales + 32 * groups;
    m.v_params = m.k_zeros + 32 * groups;
    m.bytes = m.v_params + 64 * groups;
    return m;
}

// One call's sequences and the pool (members of whole words only).
struct CacheView {
    uint8_t *pages;
    const int *new_start, *tokens, *block_table;
    const unsigned long long *mask;            // null: consecutive tokens
    int *status;
    long long table_stride, page_bytes;
    long long rows;                            // rows that the caller's tensors have
    int mask_words;
    int heads, page_shift, num_pages;          // page_shift: log2(block_tokens)
    int max_new, max_tokens;
};

struct Sequence {
    int row0, fresh, tokens;                   // first new row, new rows, tokens with the new ones
};

// Whether a sequence's numbers fit the call.  (Its new rows as an unsigned number: a start near the limits of an int makes it large.)
__device__ __forceinline__ bool fits(const CacheView &c, const Sequence &q)
{
    return q.row0 >= 0 && (unsigned)q.fresh <= (unsigned)c.max_new && (long long)q.row0 + q.fresh <= c.rows && q.tokens >= q.fresh &&
           q.tokens <= c.max_tokens;
}
// Sequence s (the same in all lanes), with nothing in it where its numbers do not fit (reported).
__device__ __forceinline__ Sequence sequence_of(const CacheView &c, int s)
{
    Sequence q;
    q.row0 = __builtin_amdgcn_readfirstlane(c.new_start[s]);
    q.fresh = __builtin_amdgcn_readfirstlane((int)((unsigned)c.new_start[s + 1] - (unsigned)q.row0));
    q.tokens = __builtin_amdgcn_readfirstlane(c.tokens[s]);
    if (!fits(c, q)) {
        if (threadIdx.x == 0) atomicOr(c.status + s, 32 /* KVC_DEV_BAD_ROW */);
        q.fresh = q.tokens = 0;
    }
    return q;
}

// The page that holds granule j of sequence s; below zero (and reported) where the table has none.
__device__ __forceinline__ int page_of(const CacheView &c, int s, long long j)
{
    const int page = c.block_table[(long long)s * c.table_stride + (j >> (c.page_shift - 4))];
    return (unsigned)page < (unsigned)c.num_pages ? page : -1;
}
// Offset of granule j of a head inside the pool.
__device__ __forceinline__ long long granule_at(const CacheView &c, int page, long long j, int head, int granule_bytes)
{
    const int in_page = (int)j & ((1 << (c.page_shift - 4)) - 1);
    return (long long)page * c.page_bytes + (long long)((head << (c.page_shift - 4)) + in_page) * granule_bytes;
}

// Byte offsets of a row's pieces inside its granule: token t (0..15), octet col of channels (8 col ...).
template <int BITS> __device__ __forceinline__ int k_code_at(int t, int col)
{
    const int g = col >> 2, q = col & 3;
    return BITS == 4 ? t * 64 + q * 16 + g * 4 : (g >> 1) * 1024 + t * 64 + q * 16 + (g & 1) * 8;
}
__device__ __forceinline__ int v_code_at(int t, int col) { return ((t >> 2) * 16 + col) * 16 + (t & 3) * 4; }    // (+ 1024: second half)
template <int GROUPS> __device__ __forceinline__ int k_scale_at(int t, int g) { return ((t >> 2) * GROUPS + g) * 8 + (t & 3) * 2; }
template <int GROUPS> __device__ __forceinline__ int k_zero_at(int t, int g) { return (t * GROUPS + g) * 2; }
template <int GROUPS> __device__ __forceinline__ int v_param_at(int t, int g) { return ((t >> 2) * GROUPS + g) * 16 + (t & 3) * 2; }   // (+ 8: zero)

// y = H x * factor in 32 bits for a row of 128 values, 8 per lane over 16 lanes in the order of the channels.
__device__ __forceinline__ void rotate_row_f32(float x[8], float factor)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= factor;
#pragma unroll
    for (int h = 1; h < 8; h <<= 1)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!(j & h)) {
                const float a = x[j], b = x[j + h];
                x[j] = a + b;
                x[j + h] = a - b;
            }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) {
        const float sign = (lane_id() & m) ? -1.0f : 1.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf(sign, x[j], __shfl_xor(x[j], m, 64));
    }
}

}  // namespace kvc
