// Attention over the quantised cache: o = sum_t softmax_t(scale * q . k_t) v_t for the new tokens of every sequence.
//
// Compiled once per pair of code widths (KVC_BITS = 10 * bits_k + bits_v).
//
// A row is one new token and one of the query heads that share a KV head; a workgroup has a block of rows of one KV head and a run of
// the sequence's tokens.  attend_kernel has blocks of 16 or 32 rows (HBM's rate bounds it, or latency), attend_wide_kernel of 128
// (arithmetic does); which of them a call takes goes by what its blocks take together (kvc_cache.hip: tiles_of).  Where a call has fewer blocks than the chip has room for, the tokens of long sequences
// are spread over several workgroups, whose results the last of them joins.
//
// Scores: the matrix product runs over the codes themselves, with 16 tokens as rows and 16 query rows as columns.  A code, masked
// out of its word together with a second one, is a half-precision subnormal, code * 2^-24 (or 2^-20), which the matrix
// instructions take as it is; the group's scale multiplies the product in 32 bits and the zero enters through one more product, of
// the zeros with the sums of the query's groups: sum_d q_d (code_d scale + zero) = scale sum_d q_d code_d + zero sum_d q_d.
// So a key costs a mask per two codes and no rounding.  Queries are scaled by a power of two to a maximum in [2^7, 2^8), so that the sums
// stay in the half type's range, and are half-precision numbers there: exact, but for elements 2^-17 and more below the largest, which lose
// bits (2^-28 of the largest at most); a rotated query is the sum of two half-precision parts.
// Softmax: running maximum and sum per row in 32 bits, base 2; sums are rescaled only when a maximum has grown by more than
// 2^kSlack.  A lane holds the weights of tokens 4 q ... 4 q + 3 of two granules for one row, which is the operand that the second
// product takes: nothing moves between lanes.
// Values: codes become packed half-precision integers (mask, and subtract the constant that the mask's exponent added), then
// code * scale + zero for two tokens at a time with one rounding, limited to the half type's range.
#include "kvc_cache.h"
#include "kvc_cache_internal.h"
#include "../../include/kvc.h"

namespace kvc {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 32;                    // tokens per wave and step
constexpr int kManyWaves = 4;
constexpr float kSlack = 8.0f;               // the maximum may grow by 2^8 before the sums are rescaled
constexpr float kBias = 6.0f;                // weights are kept as 2^(6 + score - maximum) <= 2^14
// A score that is not seen is kLowest before the factor, which is kept at 2^-60 or more (products stay below 2^40: scores below 2^-20
// instead of smaller ones), so it ends below -2^67 and weighs nothing beside the maximum that a row starts with.  A row whose scores
// are all below -2^60 counts as one that sees nothing.
constexpr float kLeastFactor = 0x1p-60f, kNothing = -0x1p60f;
constexpr float kLowest = -3.4028235e38f;
// With overflow of half-precision arithmetic set to end at the largest number, matrix instructions take NaN as 0 and infinities as the largest
// number.  A query that holds one has zeros in the products, is marked in LDS (a register would be held through all of the tokens), and
// its row's sum becomes NaN at the end.

// maximum and sum over the four lanes that hold one row
__device__ __forceinline__ float row_max(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A lane's places inside a granule, made once: a load is a scalar base and one of these.
template <int BITS_K, int BITS_V, int GROUP> struct LanePlaces {
    uint32_t k, v, ks, kz, vp;

    __device__ __forceinline__ void set()
    {
        constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
        constexpr int groups = kDim / GROUP;
        const uint32_t lane = lane_id(), q = lane >> 4, i = lane & 15;
        k = i * 64 + q * 16;
        v = map.v_codes + lane * 16;
        ks = map.k_scales + q * groups * 8;
        kz = map.k_zeros + i * groups * 2;
        vp = map.v_params + (q * groups + i / (GROUP / 8)) * 16;
    }
};

// What a lane loads of one granule; SCALES: the parameters of the scores too, as the products need them.
template <int BITS_K, int BITS_V, int GROUP> struct RawGranule {
    static constexpr int groups = kDim / GROUP;
    u32x4 k[BITS_K / 4], v[BITS_V / 4], vp;
    u32x2 ks[groups];                        // scales of 4 tokens
    uint32_t kz[(groups + 1) / 2];           // zeros of one token

    __device__ __forceinline__ void load_keys(const uint8_t *p, const LanePlaces<BITS_K, BITS_V, GROUP> &at)
    {
#pragma unroll
        for (int h = 0; h < BITS_K / 4; ++h) k[h] = *(const u32x4 *)(p + at.k + h * 1024u);
    }
    __device__ __forceinline__ void load_values(const uint8_t *p, const LanePlaces<BITS_K, BITS_V, GROUP> &at)
    {
#pragma unroll
        for (int h = 0; h < BITS_V / 4; ++h) v[h] = *(const u32x4 *)(p + at.v + h * 1024u);
        vp = *(const u32x4 *)(p + at.vp);
    }
    __device__ __forceinline__ void load_scales(const uint8_t *p, const LanePlaces<BITS_K, BITS_V, GROUP> &at)
    {
        if constexpr (groups == 1) ks[0] = *(const u32x2 *)(p + at.ks);
        else {
#pragma unroll
            for (int g = 0; g < groups; g += 2) {
                const u32x4 w = *(const u32x4 *)(p + at.ks + g * 8u);
                ks[g] = u32x2{w[0], w[1]};
                ks[g + 1] = u32x2{w[2], w[3]};
            }
        }
        if constexpr (groups == 4) {
            const u32x2 z = *(const u32x2 *)(p + at.kz);
            kz[0] = z[0];
            kz[1] = z[1];
        } else if constexpr (groups == 2) kz[0] = *(const uint32_t *)(p + at.kz);
        else kz[0] = *(const uint16_t *)(p + at.kz);
    }
    __device__ __forceinline__ half4 zeros() const
    {
        if constexpr (groups == 4) return __builtin_bit_cast(half4, u32x2{kz[0], kz[1]});
        else return __builtin_bit_cast(half4, u32x2{kz[0], 0u});
    }
};

// Codes of block g of 32 channels, of the lane's token: an operand of the product over channels.
template <int BITS> __device__ __forceinline__ half8 key_operand(const u32x4 *k, int g)
{
    uint32_t p[4];
    u32x2 w;
    if (BITS == 4) w = u32x2{k[0][g], 0};
    else w = u32x2{k[(g >> 1) * (BITS / 4 - 1)][2 * (g & 1)], k[(g >> 1) * (BITS / 4 - 1)][2 * (g & 1) + 1]};
    unpack8<BITS>(w, p);
    return __builtin_bit_cast(half8, u32x4{p[0], p[1], p[2], p[3]});
}

// (x & mask) | bits in one instruction (the compiler takes two, each with a literal)
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t bits)
{
    uint32_t r;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "s"(mask), "v"(bits));
    return r;
}

// Channel 8 i + c of tokens t0, t1 (the words of their octets): code * scale + zero in both halves.
template <int BITS> __device__ __forceinline__ uint32_t value_pair(uint32_t pair, int c, half2v scale, half2v zero)
{
    uint32_t bits;
    _Float16 offset;
    if (BITS == 4 && (c & 1)) {
        bits = and_or(pair, 0x00f000f0u, 0x54005400u);        // 64 + code
        offset = (_Float16)64.0f;
    } else {
        bits = BITS == 4 ? and_or(pair, 0x000f000fu, 0x64006400u) : pair | 0x64006400u;       // 1024 + code
        offset = (_Float16)1024.0f;
    }
    const half2v code = __builtin_bit_cast(half2v, bits) - half2v{offset, offset};
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(code, scale, zero));
}

// log of the sum of exp(scores), from the maximum in base 2 and the sum of weights (NaN: NaN)
__device__ __forceinline__ float lse_of(float top, float total)
{
    return total == 0.0f ? -__builtin_inff() : (top - kBias + __builtin_log2f(total)) * 0.69314718055994531f;
}

// The tokens that some row of a block of rows can see: [0, this).
__device__ __forceinline__ int tokens_seen(const CacheView &c, const Sequence &seq, int block, int rows_per_block, int per_kv)
{
    if (c.mask != nullptr) return seq.tokens;
    const int last = (int)(((long long)(block + 1) * rows_per_block - 1) / per_kv);
    return seq.tokens - seq.fresh + (last < seq.fresh ? last + 1 : seq.fresh);
}

template <int DT> __device__ __forceinline__ u32x4 pack_row(const float x[8])
{
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f32x2_t v = {x[2 * j], x[2 * j + 1]};
        if (DT == DT_F16) w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
        else w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
    }
    return w;
}

// The queries of one tile of 16 rows: column i of the products, channels 32 g + 8 q ... of block g, in the order in which unpack8 leaves
// a word's codes (at 4 bits every other pair stands for code * 2^-20 instead of 2^-24).
// ROTATE: rotated, as the sum of two parts.
template <int BITS_K, int GROUP, bool ROTATE> struct QueryTile {
    static constexpr int PARTS = ROTATE ? 2 : 1;
    half8 part[4 * PARTS];
    half4 sums;                              // of the groups, high parts in lanes q = 0, remainders in lanes q = 1
    float factor;                            // scores in base 2 = products * factor (not negative)
    int draft;                               // the row's new token

    __device__ __forceinline__ void fetch(const AttendArgs &a, const Sequence &seq, int head, int row, int rows)
    {
        const int q = lane_id() >> 4;
        const bool there = row < rows;
        draft = there ? row / a.per_kv : 0;
        const uint16_t *from = a.q + (long long)(seq.row0 + draft) * a.q_row + (long long)(head * a.per_kv + row % a.per_kv) * a.q_head + 8 * q;
#pragma unroll
        for (int g = 0; g < 4; ++g) part[g] = there ? *(const half8 *)(from + 32 * g) : half8{};
    }
    // Prepared queries through LDS: what one wave has made, for all waves of the workgroup.
    static constexpr int kPlaces = 4 * PARTS + 1;
    __device__ __forceinline__ void put(u32x4 (*to)[64]) const
    {
        const int lane = lane_id();
#pragma unroll
        for (int g = 0; g < 4 * PARTS; ++g) to[g][lane] = __builtin_bit_cast(u32x4, part[g]);
        const u32x2 s = __builtin_bit_cast(u32x2, sums);
        to[4 * PARTS][lane] = u32x4{s[0], s[1], __float_as_uint(factor), (uint32_t)draft};
    }
    __device__ __forceinline__ void get(const u32x4 (*from)[64])
    {
        const int lane = lane_id();
#pragma unroll
        for (int g = 0; g < 4 * PARTS; ++g) part[g] = __builtin_bit_cast(half8, from[g][lane]);
        const u32x4 w = from[4 * PARTS][lane];
        sums = __builtin_bit_cast(half4, u32x2{w[0], w[1]});
        factor = __uint_as_float(w[2]);
        draft = (int)w[3];
    }
    // whether the query is made of numbers
    __device__ __forceinline__ bool prepare(const AttendArgs &a)
    {
        constexpr int groups = kDim / GROUP;
        const int lane = lane_id(), q = lane >> 4;
        float x[4][8];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const u32x4 r = __builtin_bit_cast(u32x4, part[g]);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[g][e] = a.dtype == DT_F16 ? elem_f32<DT_F16>(r, e) : elem_f32<DT_BF16>(r, e);
        }
        if (ROTATE) {
            // strides 1, 2, 4 and 32, 64 inside the lane, 8 and 16 across the row's four lanes; the factor 1/16 joins the scores'
#pragma unroll
            for (int h = 1; h < 8; h <<= 1)
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!(e & h)) {
                            const float u = x[g][e], w = x[g][e + h];
                            x[g][e] = u + w;
                            x[g][e + h] = u - w;
                        }
#pragma unroll
            for (int h = 1; h < 4; h <<= 1)
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!(g & h)) {
                            const float u = x[g][e], w = x[g + h][e];
                            x[g][e] = u + w;
                            x[g + h][e] = u - w;
                        }
#pragma unroll
            for (int h = 16; h < 64; h <<= 1) {
                const float sign = (lane & h) ? -1.0f : 1.0f;
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[g][e] = __builtin_fmaf(sign, x[g][e], __shfl_xor(x[g][e], h, 64));
            }
        }
        float top = 0.0f;
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[g][e]));
        top = row_max(top);
        int power = (int)(__float_as_uint(top) >> 23) - 127;                 // 2^power <= top < 2^(power + 1)
        power = top == 0.0f ? 7 : power < -119 ? -119 : power;               // (both powers below are normal numbers)
        float down = __uint_as_float((uint32_t)(127 + 7 - power) << 23);
        // (log2(e) last: the scale times it may be beyond the largest number)
        factor = fabsf(a.scale) * __uint_as_float((uint32_t)(127 + power - 7) << 23) * (ROTATE ? 0.0625f : 1.0f) * 1.44269504088896341f;
        factor = fmaxf(factor, kLeastFactor);
        if (a.scale < 0.0f) down = -down;
        float sum[4] = {0, 0, 0, 0};
        bool good = true;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = x[g][e] * down;
                sum[g * groups / 4] += y[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int pair = e >> 1, from_e = pair + 4 * (e & 1);
                const float z = BITS_K == 4 && (pair & 1) ? y[from_e] * 0.0625f : y[from_e];
                const _Float16 high = (_Float16)z;
                part[g][e] = high;
                if (PARTS == 2) part[4 * (PARTS - 1) + g][e] = (_Float16)(z - (float)high);
            }
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float total = row_sum(sum[g]);
            good = good && fabsf(total) <= 65504.0f;         // (128 numbers below 2^8, or an infinity or NaN)
            const _Float16 high = (_Float16)total;
            // column i of a 16 x 16 x 16 product: lanes of q = 0 hold the sums, of q = 1 what their rounding left
            const float low = total - (float)high;
            sums[g] = g >= groups ? (_Float16)0.0f : q == 0 ? high : q == 1 ? (_Float16)low : (_Float16)0.0f;
        }
        if (!__all(good)) {
#pragma unroll
            for (int g = 0; g < 4 * PARTS; ++g) part[g] = good ? part[g] : half8{};
            sums = good ? sums : half4{};
            factor = good ? factor : kLeastFactor;
        }
        return good;
    }
};

// Scores of one granule and tile from the codes: products per group and one of the zeros ...
template <int GROUP> struct Products {
    static constexpr int groups = kDim / GROUP;
    f32x4 dot[groups], offset;

    template <typename Query> __device__ __forceinline__ void make(const half8 key[4], half4 zeros, const Query &query)
    {
#pragma unroll
        for (int g = 0; g < groups; ++g) dot[g] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < Query::PARTS; ++p)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                dot[g * groups / 4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key[g], query.part[4 * p + g], dot[g * groups / 4], 0, 0, 0);
        offset = __builtin_amdgcn_mfma_f32_16x16x16f16(zeros, query.sums, f32x4{0, 0, 0, 0}, 0, 0, 0);
    }
    // ... and the scales in 32 bits (a half of a register each, read as it is).
    __device__ __forceinline__ void scores(const u32x2 *ks, float score[4]) const
    {
        float sum[4] = {0, 0, 0, 0};
#pragma unroll
        for (int g = 0; g < groups; ++g) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum[e] = __builtin_fmaf((float)__builtin_bit_cast(half2v, (uint32_t)ks[g][e >> 1])[e & 1], dot[g][e], sum[e]);
            __builtin_amdgcn_sched_barrier(0x7fe);           // (four sums in turn: nothing but vector arithmetic stays in place)
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) score[e] = __builtin_fmaf(sum[e], 16777216.0f, offset[e]);
    }
};

// Running softmax of one tile: maximum (base 2, the same in the row's four lanes), sum of weights, and the sums of weighted values,
// channel 32 q + 8 e + ch of row i in out[ch][e].
// PARTS = 2: weights enter the products as the sum of two numbers, and their sum is a product with ones (every element has the
// row's sum); with one part that sum would be one of rounded weights, so the lanes add theirs in 32 bits (norm[0]).
template <int PARTS> struct RowState {
    float top;
    f32x4 norm, out[8];

    __device__ __forceinline__ void clear()
    {
        top = kNothing;
        norm = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int ch = 0; ch < 8; ++ch) out[ch] = f32x4{0, 0, 0, 0};
    }
    // the row's sum of weights: NaN where its query or its scores are beyond 32 bits, 0 where it sees nothing
    __device__ __forceinline__ float total(bool lost) const
    {
        const float sum = PARTS == 2 ? norm[0] : row_sum(norm[0]);
        return (lost && sum != 0.0f) || top > 3.4028235e38f ? __builtin_nanf("") : sum;
    }
    // Weights of 32 tokens.
    __device__ __forceinline__ void weigh(const float score[8], float factor, half8 weight[PARTS])
    {
        float most = kLowest;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, score[e]);
        if (__any(most * factor > top + kSlack)) {
            const float next = fmaxf(row_max(most * factor), top), shrink = __builtin_amdgcn_exp2f(top - next);
            top = next;
            norm *= shrink;
#pragma unroll
            for (int ch = 0; ch < 8; ++ch) out[ch] *= shrink;
        }
        const float down = kBias - top, one_f32 = opaque_one();
        constexpr _Float16 one = (_Float16)1.0f;
        constexpr half8 ones = {one, one, one, one, one, one, one, one};
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const f32x2_t w = {__builtin_amdgcn_exp2f(__builtin_fmaf(score[e], factor, down)),
                               __builtin_amdgcn_exp2f(__builtin_fmaf(score[e + 1], factor, down))};
            const half2v high = __builtin_convertvector(w, half2v);
            weight[0][e] = high[0];
            weight[0][e + 1] = high[1];
            if (PARTS == 1) norm[0] += w[0] + w[1];
            else {                           // (the halves are read as they are)
                const f32x2_t rest = {__builtin_fmaf((float)high[0], -one_f32, w[0]), __builtin_fmaf((float)high[1], -one_f32, w[1])};
                const half2v low = __builtin_convertvector(rest, half2v);
                weight[PARTS - 1][e] = low[0];
                weight[PARTS - 1][e + 1] = low[1];
            }
        }
        if (PARTS == 1) return;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) norm = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, weight[p], norm, 0, 0, 0);
    }
    __device__ __forceinline__ void add(int ch, half8 values, const half8 &weight)
    {
        out[ch] = __builtin_amdgcn_mfma_f32_16x16x32_f16(values, weight, out[ch], 0, 0, 0);
    }
};

// Which of the 32 tokens from number j0 of the new ones on (or before them: j0 > -32) a new token sees: all before the new ones, then its
// mask's bits, or itself and those before it.
__device__ __forceinline__ uint32_t seen_bits(const CacheView &c, const Sequence &seq, int draft, int j0)
{
    if (j0 <= -32) return ~0u;
    uint32_t bits;
    if (c.mask == nullptr) {
        const int n = draft - j0 + 1;
        bits = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
    } else {
        // (the word behind the last is not there; what it would hold is behind the sequence's last token)
        const unsigned long long *row = c.mask + (long long)(seq.row0 + draft) * c.mask_words;
        const int from = j0 < 0 ? 0 : j0, word = from >> 6, shift = from & 63;
        unsigned long long w = word < c.mask_words ? row[word] >> shift : 0ull;
        if (shift > 32 && word + 1 < c.mask_words) w |= row[word + 1] << (64 - shift);
        bits = (uint32_t)w;
        if (j0 < 0) bits = bits << -j0 | ((1u << -j0) - 1u);
    }
    return bits;
}

// Scores of what a row does not see, of the 32 tokens from `token` on, become the lowest number.
__device__ __forceinline__ void only_seen(float score[8], const CacheView &c, const Sequence &seq, int draft, int token, int past, int end,
                                          const bool there[2])
{
    const int q = lane_id() >> 4, left = end - token;
    uint32_t bits = seen_bits(c, seq, draft, token - past);
    if (left < 32) bits &= left <= 0 ? 0u : (1u << left) - 1u;
    if (!there[0]) bits &= 0xffff0000u;
    if (!there[1]) bits &= 0x0000ffffu;
    bits >>= 4 * q;
#pragma unroll
    for (int e = 0; e < 8; ++e) score[e] = (bits >> (16 * (e >> 2) + (e & 3))) & 1u ? score[e] : kLowest;
}

// Values of zero for the tokens of a granule that are not there: what lies behind the end may be anything.
__device__ __forceinline__ u32x4 only_there(u32x4 vp, bool page, int first_token, int tokens)
{
    const int q = lane_id() >> 4;
    uint32_t keep[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) keep[e] = page && first_token + 4 * q + e < tokens ? 0xffffu : 0u;
    const uint32_t low = keep[0] | keep[1] << 16, high = keep[2] | keep[3] << 16;
    return u32x4{vp[0] & low, vp[1] & high, vp[2] & low, vp[3] & high};
}

// Operands of the product over tokens for channels 8 i + ch, two at a time (what follows on a product has another one in between):
// f(ch, operand of ch, operand of ch + 1), ch even.
template <int BITS_V, typename Raw, typename F> __device__ __forceinline__ void value_operands(const Raw *r, F f)
{
#pragma unroll
    for (int ch = 0; ch < 8; ch += 2) {
        u32x4 w[2];
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int word = BITS_V == 4 ? 0 : ch >> 2, byte = BITS_V == 4 ? ch >> 1 : (ch + which) & 3;
                const uint32_t pair = __builtin_amdgcn_perm(r[e >> 1].v[word][2 * (e & 1) + 1], r[e >> 1].v[word][2 * (e & 1)],
                                                            0x0c040c00u + (uint32_t)byte * 0x00010001u);
                w[which][e] = value_pair<BITS_V>(pair, ch + which, __builtin_bit_cast(half2v, (uint32_t)r[e >> 1].vp[e & 1]),
                                                 __builtin_bit_cast(half2v, (uint32_t)r[e >> 1].vp[2 + (e & 1)]));
            }
        f(ch, __builtin_bit_cast(half8, w[0]), __builtin_bit_cast(half8, w[1]));
    }
}

// Pages of a wave's coming steps of 32 tokens: step n is granules first + 2 (WAVES n + wave) and the one behind it.
template <int WAVES> struct PageWindow {
    int entries, ahead;                      // lane l: the page of granule l & 1 of step ahead + (l >> 1)

    __device__ __forceinline__ void start() { ahead = -32; }
    // granule h of step n; n goes up by one from call to call (both granules of a step)
    __device__ __forceinline__ int page(const CacheView &c, int s, int first, int wave, int last, int n, int h)
    {
        if (n == ahead + 32) {
            ahead = n;
            const int lane = lane_id(), j = first + 2 * (WAVES * (n + (lane >> 1)) + wave) + (lane & 1);
            entries = page_of(c, s, j < last ? j : last);        // (behind the end: the last one's page, and a place in it)
            if (entries < 0) atomicOr(c.status + s, KVC_DEV_BAD_BLOCK);
        }
        return __builtin_amdgcn_readlane(entries, 2 * (n - ahead) + h);
    }
};

// ---- which tokens of which sequence a workgroup has ---------------------------------------------------

// A part of a sequence: `count` parts of `chunk` tokens each, this is number `index`.  Parts of a sequence with several of them leave
// their results in slots slot0 ... slot0 + count - 1 (times the heads and blocks of rows).
struct Part {
    int s, index, count, slot0;
    long long chunk;
};

// Sum over the wave's lanes up to and with this one.
__device__ __forceinline__ unsigned sum_upto(unsigned x)
{
    // inside rows of 16, then the last lanes of the rows before (two steps)
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);       // row_shr:1
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);       // row_shr:2
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);       // row_shr:4
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);       // row_shr:8
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);       // row_bcast:15
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);       // row_bcast:31
    return x;
}
__device__ __forceinline__ float max_of_row(float x)         // over the 16 lanes
{
    x = fmaxf(x, dpp_f32<DPP_QUAD_XOR1>(x));
    x = fmaxf(x, dpp_f32<DPP_QUAD_XOR2>(x));
    x = fmaxf(x, dpp_f32<DPP_HALF_MIRROR>(x));
    return fmaxf(x, dpp_f32<DPP_MIRROR>(x));
}
__device__ __forceinline__ float sum_of_row(float x)
{
    x += dpp_f32<DPP_QUAD_XOR1>(x);
    x += dpp_f32<DPP_QUAD_XOR2>(x);
    x += dpp_f32<DPP_HALF_MIRROR>(x);
    return x + dpp_f32<DPP_MIRROR>(x);
}

// Part u of the call, in all waves.  The lengths are on the device, so the division is made here, from the lengths of up to 256 sequences
// in units of STEP tokens.  The measure is a piece length: the shortest with which the pieces of all sequences fit the chip at
// once (per head and block of rows); or, with more sequences than that, twice an even share, so that only the longest are cut.
// Where two workgroups share a compute unit each is slower for it (by a.alone), so that up to that much longer pieces with which
// every workgroup has a unit of its own are better.
// A sequence is then cut into equal pieces of that length at most; nothing is cut where that would save less than joining costs
// (a.joining units).  With more than 256 sequences a piece is a whole one.  False: there is no part u, or nothing in it.
template <int STEP> __device__ __forceinline__ bool find_part(const AttendArgs &a, int u, Part &p, Sequence &seq)
{
    const CacheView &c = a.c;
    if (!a.divide) {
        if (u >= a.n) return false;
        p = Part{u, 0, 1, 0, 1ll << 40};
        seq = sequence_of(c, u);
        return true;
    }
    const int lane = lane_id();
    Sequence of[4];
    int units[4], busy = 0, longest = 0;
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        units[k] = 0;
        if (64 * k < a.n) {
            const int s = 64 * k + lane;
            if (s < a.n) {
                of[k].row0 = c.new_start[s];
                of[k].fresh = (int)((unsigned)c.new_start[s + 1] - (unsigned)of[k].row0);
                of[k].tokens = c.tokens[s];
                const bool fit = fits(c, of[k]);
                if (fit && of[k].fresh) units[k] = (int)(((unsigned)of[k].tokens + STEP - 1u) / STEP);
                if (!fit && blockIdx.x == 0 && threadIdx.x < 64) atomicOr(c.status + s, KVC_DEV_BAD_ROW);     // (no workgroup comes to it)
            }
            sum += (float)units[k];
            longest = units[k] > longest ? units[k] : longest;
            busy += __popcll(__ballot(units[k] > 0));
        }
    }
    if (busy == 0) return false;
    longest = __builtin_amdgcn_readfirstlane((int)row_max(max_of_row((float)longest)));
    // in units; joining takes time by the number of pieces, so that piece + a.joining_piece * longest / piece is to be small
    const int least = __builtin_amdgcn_readfirstlane((int)__builtin_amdgcn_sqrtf(a.joining_piece * (float)longest)) + 1;
    if (a.n > 1) sum = row_sum(sum_of_row(sum));
    // the shortest piece from there on with which there are no more than `parts`
    auto shortest = [&](int parts) {
        if (longest <= least) return least;
        if (a.n == 1) {
            const int even = (longest + parts - 1) / parts;
            return even > least ? even : least;
        }
        // between an even share and one that leaves room for a shorter last piece of every sequence, by bisection
        int piece = __builtin_amdgcn_readfirstlane((int)(sum * 0.9999f / (float)parts)), most = longest;
        piece = piece > least ? piece : least;
        if (busy < parts) {
            const int roomy = __builtin_amdgcn_readfirstlane((int)(sum * 1.0001f / (float)(parts - busy))) + 1;
            most = roomy < most ? roomy : most;
        }
        while (piece < most) {
            const int middle = (piece + most) >> 1;
            float made = 0.0f;               // (below 2^24: exact)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (64 * k < a.n) made += (float)(((unsigned)units[k] + (unsigned)middle - 1u) / (unsigned)middle);
            if (row_sum(sum_of_row(made)) <= (float)parts) most = middle;
            else piece = middle + 1;
        }
        return piece;
    };
    int piece;
    if (busy > a.parts) {
        piece = __builtin_amdgcn_readfirstlane((int)(2.0f * sum / (float)a.parts)) + 1;
        piece = piece > least ? piece : least;
    } else {
        piece = shortest(a.parts);
        if (a.alone > 0.0f && 2 * busy <= a.parts) {
            const int longer = shortest(a.parts / 2);
            if ((float)longer <= a.alone * (float)piece) piece = longer;
        }
    }
    if (piece + a.joining > longest) piece = longest;
    // pieces of the sequences before, and slots of those of them that are cut (both below 2^16)
    unsigned before = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (64 * k < a.n) {
            const unsigned parts = units[k] ? ((unsigned)units[k] + (unsigned)piece - 1u) / (unsigned)piece : 0u;
            const unsigned upto = before + sum_upto(parts | (parts > 1 ? parts << 16 : 0u));
            const unsigned long long behind = __ballot((int)(upto & 0xffffu) > u);
            if (behind) {
                const int owner = __builtin_ctzll(behind);
                const unsigned mine = __builtin_amdgcn_readlane((int)parts, owner), end = __builtin_amdgcn_readlane((int)upto, owner);
                const unsigned whole = __builtin_amdgcn_readlane(units[k], owner);
                p.s = 64 * k + owner;
                p.count = (int)mine;
                p.index = u - (int)((end & 0xffffu) - mine);
                p.slot0 = (int)((end >> 16) - (mine > 1 ? mine : 0u));
                p.chunk = (long long)((whole + mine - 1) / mine) * STEP;
                seq.row0 = __builtin_amdgcn_readlane(of[k].row0, owner);
                seq.fresh = __builtin_amdgcn_readlane(of[k].fresh, owner);
                seq.tokens = __builtin_amdgcn_readlane(of[k].tokens, owner);
                return true;
            }
            before = __builtin_amdgcn_readlane((int)upto, 63);
        }
    }
    return false;
}

// Where a part that starts at token `begin` ends.  Granules whose page the table does not have are read from page 0 in their place, so a
// pool without pages has no tokens to be read (reported).
__device__ __forceinline__ int end_of(const CacheView &c, int s, const Part &part, int begin, int limit)
{
    if (c.num_pages == 0) {
        if (threadIdx.x == 0) atomicOr(c.status + s, KVC_DEV_BAD_BLOCK);
        return begin;
    }
    return begin + part.chunk < limit ? (int)(begin + part.chunk) : limit;
}

// ---- results of several workgroups --------------------------------------------------------------------

// What workgroups leave for each other are pairs of numbers, stored as single words of agent scope: such a store goes through to memory,
// and loads of that scope (bit 4 of a buffer load's last argument, sc1) pass by what the XCD's own L2 may have.
// (A release of agent scope writes back a whole L2 per workgroup, 139 instead of 45 us for one token over 128k, and an acquire
// takes 1.5 to 2.5 us.)
__device__ __forceinline__ void leave(float *p, float a, float b)
{
    const unsigned long long v = (unsigned long long)__float_as_uint(a) | (unsigned long long)__float_as_uint(b) << 32;
    __hip_atomic_store((unsigned long long *)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

struct LeftRows {
    __amdgpu_buffer_rsrc_t words;

    __device__ __forceinline__ LeftRows(const float *p, long long floats)
    {
        words = __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)(unsigned)(floats * 4), 0x27000);
    }
    __device__ __forceinline__ f32x4 four(unsigned at) const
    {
        return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(words, (int)(at * 4u), 0, 16));
    }
    __device__ __forceinline__ f32x2_t two(unsigned at) const
    {
        return __builtin_bit_cast(f32x2_t, __builtin_amdgcn_raw_buffer_load_b64(words, (int)(at * 4u), 0, 16));
    }
};

// True in all threads of the workgroup that is the last of `count` to get here (the counter is left at zero, as it was found).  What all
// of them have left before is then there to be taken: every wave waits for its stores to arrive before the workgroup counts.
__device__ __forceinline__ bool last_to_arrive(int *counter, int count)
{
    __shared__ int order;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) order = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (order != count - 1) return false;
    asm volatile("" ::: "memory");           // (nothing is loaded before this)
    if (threadIdx.x == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}

// Channels that lane i of sixteen has of a row that it leaves: pairs 2 i + 32 j, j = 0..3, so that the lanes' pairs lie next to each
// other.
constexpr int pair_at(int i, int j) { return 2 * i + 32 * j; }

// Joins the parts of `rows` query rows (128 at most): part k of row r has its sums at (first + k * stride + r) * kDim of `part` and
// (maximum, sum of weights) at twice that place of `ml`.  Sixteen lanes with eight channels each per row, or several times
// sixteen that take turns with the parts, eight parts requested at a time, the first together with the maxima; `space` is LDS
// for every sixteen lanes.  done(row, i, values of channels 8 i ..., maximum, sum).
template <int THREADS, typename F>
__device__ __forceinline__ void join_parts(const LeftRows &part, const LeftRows &ml, unsigned first, unsigned stride, int rows, int count,
                                           float (*space)[kDim + 4], F done)
{
    constexpr int sets = THREADS / 16;
    const int set = (int)threadIdx.x >> 4, i = (int)threadIdx.x & 15;
    int side = 1;                            // rows at a time: a power of two
    while (side < rows && 2 * side <= sets) side *= 2;
    const int per_row = sets / side;         // (sets beyond side * per_row do nothing)
    for (int base = 0; base < rows; base += side) {
        const int r = base + set % side, turn = set / side;
        const bool mine = r < rows && turn < per_row && turn < count;
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, highest = kLowest, total = 0.0f;
        f32x2_t s[8];
        f32x4 lo[8], hi[8];
        // (part turn + n * per_row for n = n0 ... n0 + 7; turns behind the last part take that one, and no share of it)
        auto request = [&](int n0) {
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                if ((n0 + n) * per_row >= count) break;
                const int k = turn + (n0 + n) * per_row < count ? turn + (n0 + n) * per_row : count - 1;
                const unsigned at = first + (unsigned)k * stride + (unsigned)r;
                s[n] = ml.two(2 * at);
                lo[n] = part.four(at * kDim + 8 * i);
                hi[n] = part.four(at * kDim + 8 * i + 4);
            }
        };
        if (mine) {
            request(0);
            // sixteen lanes look at sixteen parts at a time
#pragma unroll 4
            for (int k = i; k < count; k += 16) highest = fmaxf(highest, ml.two(2 * (first + (unsigned)k * stride + (unsigned)r))[0]);
        }
        highest = max_of_row(highest);
        if (mine) {
            for (int n0 = 0; n0 * per_row < count; n0 += 8) {
                if (n0) request(n0);
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    if ((n0 + n) * per_row >= count) break;
                    const float share = turn + (n0 + n) * per_row < count ? __builtin_amdgcn_exp2f(s[n][0] - highest) : 0.0f;
                    total = __builtin_fmaf(s[n][1], share, total);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = __builtin_fmaf(lo[n][e], share, x[e]);
                        x[4 + e] = __builtin_fmaf(hi[n][e], share, x[4 + e]);
                    }
                }
            }
        }
        if (per_row > 1) {                   // (the same in all threads)
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) space[set][8 * i + e] = x[e];
            if (i == 0) space[set][kDim] = total;
            __syncthreads();
            if (turn == 0) {
                for (int k = 1; k < per_row; ++k) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] += space[set + k * side][8 * i + e];
                    total += space[set + k * side][kDim];
                }
            }
        }
        if (mine && turn == 0) done(r, i, x, highest, total);
    }
}

// The same where there are as many rows as sets of sixteen lanes or more, and 16 / M parts or fewer: a set has M rows at a time, all of
// whose parts are requested together.
template <int THREADS, int M, typename F>
__device__ __forceinline__ void join_few_parts(const LeftRows &part, const LeftRows &ml, unsigned first, unsigned stride, int rows, int count, F done)
{
    constexpr int sets = THREADS / 16, most = 16 / M;
    const int set = (int)threadIdx.x >> 4, i = (int)threadIdx.x & 15;
    for (int base = 0; base < rows; base += sets * M) {
        f32x2_t s[M][most];
        f32x4 lo[M][most], hi[M][most];
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int k = 0; k < most; ++k) {
                if (k >= count) break;
                const int row = base + m * sets + set < rows ? base + m * sets + set : rows - 1;
                const unsigned at = first + (unsigned)k * stride + (unsigned)row;
                s[m][k] = ml.two(2 * at);
                lo[m][k] = part.four(at * kDim + 8 * i);
                hi[m][k] = part.four(at * kDim + 8 * i + 4);
            }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            float x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, highest = kLowest, total = 0.0f;
#pragma unroll
            for (int k = 0; k < most; ++k) {
                if (k >= count) break;
                highest = fmaxf(highest, s[m][k][0]);
            }
#pragma unroll
            for (int k = 0; k < most; ++k) {
                if (k >= count) break;
                const float share = __builtin_amdgcn_exp2f(s[m][k][0] - highest);
                total = __builtin_fmaf(s[m][k][1], share, total);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = __builtin_fmaf(lo[m][k][e], share, x[e]);
                    x[4 + e] = __builtin_fmaf(hi[m][k][e], share, x[4 + e]);
                }
            }
            if (base + m * sets + set < rows) done(base + m * sets + set, i, x, highest, total);
        }
    }
}

// Where the results of a block of query rows go.
struct Results {
    const AttendArgs &a;
    const Sequence &seq;
    int head, first;

    __device__ __forceinline__ uint16_t *row(int row, int &d, int &query_head) const
    {
        d = (first + row) / a.per_kv;
        query_head = head * a.per_kv + (first + row) % a.per_kv;
        return a.out + (long long)(seq.row0 + d) * a.o_row + (long long)query_head * a.o_head;
    }
    __device__ __forceinline__ void lse(int d, int query_head, float highest, float total) const
    {
        if (a.lse) a.lse[(long long)(seq.row0 + d) * (a.c.heads * a.per_kv) + query_head] = lse_of(highest, total);
    }
    // eight channels in a row; `speaks`: the lane writes the row's lse
    template <int DT> __device__ __forceinline__ void octet(int r, int channel, const float x[8], bool speaks, float highest, float total) const
    {
        int d, query_head;
        uint16_t *to = row(r, d, query_head);
        const float share = total == 0.0f ? 0.0f : 1.0f / total;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e] * share;
        *(u32x4 *)(to + channel) = pack_row<DT>(y);
        if (speaks) lse(d, query_head, highest, total);
    }
};

// ---- few rows: the waves of a workgroup share rows and divide tokens --------------------------------

// One block of 16 * TILES rows, whose queries are in the registers of every wave; the waves take 32 tokens
// at a time in turn and their results meet in LDS at the end.  So a code is read once per block, straight into the registers of the one
// wave that uses it: with few rows a token brings 160 to 300 bytes per head and 512 operations per row, and HBM is the bound.
// One token over 128k (8 KV heads, 4 query heads each, 4 bits, groups of 32, fp16; 168 MB): 41.5 us, 4.1 TB/s; what more tokens cost,
// 5.5 TB/s (pure reads past the caches reach 7.0, and why these do not is not known), and some 11 us do not depend on them: dividing (1.5), pages and queries (3), the waves' join
// (2), the workgroups' join (4 to 5).  Vector instructions take 45 % of the time there, matrix instructions 17 %.  4 sequences of 16k to
// 32k tokens, 8-bit K, groups of 128 (92 MB): 25.2 us.  One token over 1k: 10.9 us, latencies one after the other and one compute unit's
// arithmetic per head.
// Two tiles per block, 64 drafts over 16k tokens, 4 query heads: 45 us, in blocks of 16 rows 54, of 128 71; 24 drafts over 2k 15.7, in blocks
// of 16 13.9.
// As many waves as the registers leave room for in a compute unit, three per SIMD or two: what is in flight is what hides the memory's
// latency, one step's codes per wave.  (Four waves and three workgroups per unit: more pieces to join.  Eight waves with one / two / three steps
// in flight: 19.1 / 18.7 / 19.0 us for 32 sequences of 0.5 to 2k tokens, twelve with one 17.5; sixteen spill.)  Two
// tiles of rotated queries do not fit in full: 36 to 108 bytes per lane are held in memory with groups of 32, up to 32 with larger ones, and up to
// twelve registers per 32 tokens come from there.
constexpr int few_waves(int tiles, bool rotate) { return tiles == 1 && !rotate ? 12 : 8; }

template <int BITS_K, int BITS_V, int GROUP, int TILES, bool ROTATE, int PARTS>
__global__ __launch_bounds__(64 * few_waves(TILES, ROTATE), few_waves(TILES, ROTATE) / 4) void attend_kernel(AttendArgs a)
{
    constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
    constexpr int waves = few_waves(TILES, ROTATE);
    typedef RawGranule<BITS_K, BITS_V, GROUP> Raw;
    __shared__ __attribute__((aligned(16))) float sums[waves][16][kDim + 4];
    __shared__ float tops[waves][16 * TILES], norms[waves][16 * TILES];
    __shared__ int lost[16 * TILES];         // rows whose queries are no numbers

    const CacheView &c = a.c;
    const int lane = lane_id(), wave = wave_id(), q = lane >> 4, i = lane & 15;
    const int each = c.heads * a.row_blocks, u = (int)(blockIdx.x / (unsigned)each), rest = (int)(blockIdx.x % (unsigned)each);
    const int head = rest % c.heads, block = rest / c.heads;
    Part part;
    Sequence seq;
    if (!find_part<kStep * waves>(a, u, part, seq)) return;
    const int s = part.s;
    const int first = block * 16 * TILES, rows = seq.fresh * a.per_kv;
    if (first >= rows) return;
    const int limit = tokens_seen(c, seq, block, 16 * TILES, a.per_kv), past = seq.tokens - seq.fresh;
    const int count = (int)((limit + part.chunk - 1) / part.chunk);      // (of this block of rows)
    if (part.index >= count) return;
    const int begin = (int)(part.index * part.chunk), end = end_of(c, s, part, begin, limit);

    // overflow of half-precision arithmetic ends at 65504 instead of infinity (bit 23 of the mode register)
    __builtin_amdgcn_s_setreg((0 << 11) | (23 << 6) | 1, 1);

    // ---- tokens: the wave's step n is 32 tokens from begin + 32 * (waves * n + wave); the first are requested before the queries
    const int steps = (end - begin + kStep - 1) / kStep;
    const int mine = steps > wave ? (steps - wave + waves - 1) / waves : 0;
    LanePlaces<BITS_K, BITS_V, GROUP> at;
    at.set();
    PageWindow<waves> window;
    window.start();
    // The granules of a step: where they are, and whether their pages are there.
    struct Step {
        const uint8_t *at[2];
        bool there[2];
    };
    auto find = [&](int n) {
        Step f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int page = window.page(c, s, begin >> 4, wave, (end - 1) >> 4, n, h);
            f.there[h] = page >= 0;
            f.at[h] = c.pages + granule_at(c, page < 0 ? 0 : page, (begin >> 4) + 2 * (waves * n + wave) + h, head, map.bytes);
        }
        return f;
    };
    auto load_keys = [&](Raw *r, const Step &f) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            r[h].load_keys(f.at[h], at);
            r[h].load_scales(f.at[h], at);
        }
    };
    auto load_values = [&](Raw *r, const Step &f) {
#pragma unroll
        for (int h = 0; h < 2; ++h) r[h].load_values(f.at[h], at);
    };
    typedef QueryTile<BITS_K, GROUP, ROTATE> Query;
    static_assert(sizeof(u32x4) * 64 * Query::kPlaces * TILES <= sizeof(sums), "the queries go through the room of the sums");
    u32x4(*shared_queries)[64] = (u32x4(*)[64])sums;
    Query query[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t)
        if (wave == t) query[t].fetch(a, seq, head, first + 16 * t + i, rows);
    Raw now[2];
    Step now_at = {}, next_at = {};
    if (mine > 0) {
        now_at = find(0);
        load_keys(now, now_at);
        load_values(now, now_at);
    }
    RowState<PARTS> state[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t)
        if (wave == t) {                     // one wave per tile prepares it for all of them
            lost[16 * t + i] = !query[t].prepare(a);
            query[t].put(shared_queries + t * Query::kPlaces);
        }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        query[t].get(shared_queries + t * Query::kPlaces);
        state[t].clear();
    }
    __syncthreads();                         // (before the room is the sums' again)
    // Scores and weights of step n, from r's keys ...
    auto weigh = [&](Raw *r, const Step &f, int n, half8 (*weight)[PARTS]) {
        const int token = begin + kStep * (waves * n + wave);
        const bool all = token + kStep <= past && token + kStep <= end && f.there[0] && f.there[1];
        float score[TILES][8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            half8 key[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) key[g] = key_operand<BITS_K>(r[h].k, g);
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                Products<GROUP> products;
                products.make(key, r[h].zeros(), query[t]);
                products.scores(r[h].ks, score[t] + 4 * h);
            }
        }
        if (!all) {
#pragma unroll
            for (int t = 0; t < TILES; ++t) only_seen(score[t], c, seq, query[t].draft, token, past, end, f.there);
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t) state[t].weigh(score[t], query[t].factor, weight[t]);
    };
    // ... and its values.
    auto add = [&](Raw *r, const Step &f, int n, const half8 (*weight)[PARTS]) {
        const int token = begin + kStep * (waves * n + wave);
        if (token + kStep > seq.tokens || !f.there[0] || !f.there[1]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) r[h].vp = only_there(r[h].vp, f.there[h], token + 16 * h, seq.tokens);
        }
        value_operands<BITS_V>(r, [&](int ch, half8 v0, half8 v1) {
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    state[t].add(ch, v0, weight[t][p]);
                    state[t].add(ch + 1, v1, weight[t][p]);
                }
        });
    };
    // The next step's keys and values are requested as soon as the step's own are used: one set of registers, so that more waves fit.
    half8 weight[TILES][PARTS];
    for (int n = 0; n < mine; ++n) {
        weigh(now, now_at, n, weight);
        if (n + 1 < mine) {
            next_at = find(n + 1);
            load_keys(now, next_at);
        }
        add(now, now_at, n, weight);
        if (n + 1 < mine) {
            load_values(now, next_at);
            now_at = next_at;
        }
    }

    // ---- the waves' results: maxima and sums first, then the rows, a tile at a time
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const float total = state[t].total(lost[16 * t + i] != 0);
        if (q == 0) {
            tops[wave][16 * t + i] = state[t].top;
            norms[wave][16 * t + i] = total;
        }
    }
    __syncthreads();
    constexpr int dtype = PARTS == 2 ? DT_F16 : DT_BF16;
    const int here = rows - first < 16 * TILES ? rows - first : 16 * TILES;
    const long long slot = ((long long)(part.slot0 + part.index) * each + rest) * (16 * TILES);
    const Results results{a, seq, head, first};
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        float most = kLowest;
#pragma unroll
        for (int w = 0; w < waves; ++w) most = fmaxf(most, tops[w][16 * t + i]);
        const float share = __builtin_amdgcn_exp2f(state[t].top - most);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4 v;
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) v[ch] = state[t].out[4 * half + ch][e] * share;
                *(f32x4 *)&sums[wave][i][32 * q + 8 * e + 4 * half] = v;
            }
        __syncthreads();
        // sixteen lanes have one row, 8 channels each
        const int r = (int)threadIdx.x >> 4, row = 16 * t + r;
        if (r < 16 && row < here) {
            float x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, total = 0.0f, highest = kLowest;
#pragma unroll
            for (int w = 0; w < waves; ++w) highest = fmaxf(highest, tops[w][row]);
#pragma unroll
            for (int w = 0; w < waves; ++w) total += norms[w][row] * __builtin_amdgcn_exp2f(tops[w][row] - highest);
            if (count == 1) {
#pragma unroll
                for (int w = 0; w < waves; ++w) {
                    const f32x4 lo = *(const f32x4 *)&sums[w][r][8 * i], hi = *(const f32x4 *)&sums[w][r][8 * i + 4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] += lo[e];
                        x[4 + e] += hi[e];
                    }
                }
                results.octet<dtype>(row, 8 * i, x, i == 0, highest, total);
            } else {
#pragma unroll
                for (int w = 0; w < waves; ++w)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const f32x2_t v = *(const f32x2_t *)&sums[w][r][pair_at(i, j)];
                        x[2 * j] += v[0];
                        x[2 * j + 1] += v[1];
                    }
#pragma unroll
                for (int j = 0; j < 4; ++j) leave(a.part + (slot + row) * kDim + pair_at(i, j), x[2 * j], x[2 * j + 1]);
                if (i == 0) leave(a.part_ml + 2 * (slot + row), highest, total);
            }
        }
        if (t + 1 < TILES) __syncthreads();
    }
    if (count == 1) return;
    const unsigned first_slot = (unsigned)(part.slot0 * each + rest) * (16 * TILES);
    if (!last_to_arrive(a.counters + (long long)part.slot0 * each + rest, count)) return;
    join_parts<64 * waves>(LeftRows(a.part, a.part_rows * kDim), LeftRows(a.part_ml, a.part_rows * 2), first_slot, (unsigned)each * 16 * TILES, here, count,
                               (float(*)[kDim + 4])sums, [&](int r, int lane_of, const float x[8], float highest, float total) {
                                   results.octet<dtype>(r, 8 * lane_of, x, lane_of == 0, highest, total);
                               });
}

// ---- many rows: the waves of a workgroup share tokens and divide rows --------------------------------

// 128 rows, 32 for each of four waves.  128 tokens at a time: each wave turns 32 of them into operands, which go through LDS in the
// order of the lanes (every access is one KB in a row: no bank conflicts), so masking codes and restoring values, some 200 vector
// instructions per 32 tokens, is done once for 128 rows and not once per wave.
// Arithmetic bounds it: per wave and 32 tokens 36 matrix instructions (16 of 16 x 16 x 32 for the scores, 4 smaller ones for the zeros, 16
// for the values; a second part of rotated queries adds 16, of the weights for fp16 results 20) and some 180 (bf16, groups of 64) to
// 250 (fp16, groups of 32) of vector arithmetic: scales and zeros 48 or 80, 16 exponentials and their arguments, the sums, the
// second parts, a quarter of the operands' making.  Two waves of a SIMD get little from each other: 16 products
// and 64 multiply-adds of each take 226 and 159 ns alone, 399 one kind after the other in both waves, 392 with four multiply-adds behind
// every product, and 470 (twice 235) where one wave has all the products and the other all the multiply-adds; only exponentials run
// beside products for nothing.
// 512 new tokens behind 32k (8 x 8 heads, 8 bits, groups of 64, bf16; 545 GFLOP): 690 us, 790 TFLOP/s (a large library product:
// 1135; fp16, with weights in two parts, 857), vector instructions 56 % of the time and matrix instructions 40 %; trees of 64 drafts over
// 8 x 8k (rotated 4 bits, groups of 32, fp16; 137 GFLOP, 275 with the second parts): 285 us, 46 % and 51 %.
// Two workgroups per compute unit, as 256 registers per lane allow.  Not all fits: with rotated queries 84 to 156 bytes per lane are held
// in memory (groups of 64 24 to 116, of 128 up to 60), without up to 20, nearly all of them numbers of the beginning, the next load and
// the end; among the products of 32 tokens up to four registers come from there.  The scores of the next 32
// tokens ahead of this one's weights gained nothing, nor did two steps of the loop at once.
template <int BITS_K, int BITS_V, int GROUP, bool ROTATE, int PARTS>
__global__ __launch_bounds__(64 * kManyWaves, 2) void attend_wide_kernel(AttendArgs a)
{
    constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
    constexpr int groups = kDim / GROUP, param_words = 16 * groups;      // words of a granule's key scales and zeros
    typedef RawGranule<BITS_K, BITS_V, GROUP> Raw;
    __shared__ u32x4 lds[2 * kManyWaves * 4 * 64 + kManyWaves * 8 * 64];
    u32x4(*keys)[4][64] = (u32x4(*)[4][64]) lds;                         // of 8 granules
    u32x4(*values)[8][64] = (u32x4(*)[8][64])(lds + 2 * kManyWaves * 4 * 64);      // of 4 steps
    __shared__ __attribute__((aligned(16))) uint32_t params[2 * kManyWaves][param_words];
    __shared__ int present[2 * kManyWaves];
    __shared__ int lost[kWideRows];          // rows whose queries are no numbers

    const CacheView &c = a.c;
    const int lane = lane_id(), wave = wave_id(), q = lane >> 4, i = lane & 15;
    const int each = c.heads * a.row_blocks, u = (int)(blockIdx.x / (unsigned)each), rest = (int)(blockIdx.x % (unsigned)each);
    const int head = rest % c.heads, block = rest / c.heads;
    Part part;
    Sequence seq;
    if (!find_part<kStep * kManyWaves>(a, u, part, seq)) return;
    const int s = part.s;
    const int first = block * kWideRows, rows = seq.fresh * a.per_kv;
    if (first >= rows) return;
    const int limit = tokens_seen(c, seq, block, kWideRows, a.per_kv), past = seq.tokens - seq.fresh;
    const int count = (int)((limit + part.chunk - 1) / part.chunk);
    if (part.index >= count) return;
    const int begin = (int)(part.index * part.chunk), end = end_of(c, s, part, begin, limit);
    __builtin_amdgcn_s_setreg((0 << 11) | (23 << 6) | 1, 1);             // (see attend_kernel)

    QueryTile<BITS_K, GROUP, ROTATE> query[2];
    RowState<PARTS> state[2];
    LanePlaces<BITS_K, BITS_V, GROUP> at;
    at.set();
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        query[t].fetch(a, seq, head, first + 32 * wave + 16 * t + i, rows);
        lost[32 * wave + 16 * t + i] = !query[t].prepare(a);
        state[t].clear();
        __builtin_amdgcn_sched_barrier(0);   // (one tile's numbers in 32 bits at a time)
    }

    const int steps = (end - begin + kStep - 1) / kStep, rounds = (steps + kManyWaves - 1) / kManyWaves;
    PageWindow<kManyWaves> window;
    window.start();
    Raw raw[2];
    uint32_t param[2];
    bool there[2] = {false, false};
    auto load = [&](int n) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int page = window.page(c, s, begin >> 4, wave, (end - 1) >> 4, n, h);
            there[h] = page >= 0;
            const uint8_t *p = c.pages + granule_at(c, page < 0 ? 0 : page, (begin >> 4) + 2 * (kManyWaves * n + wave) + h, head, map.bytes);
            raw[h].load_keys(p, at);
            raw[h].load_values(p, at);
            param[h] = *(const uint32_t *)(p + map.k_scales + (uint32_t)(lane % param_words) * 4u);
        }
    };
    if (rounds > 0) load(0);
    const bool busy = first + 32 * wave < rows;              // (a wave without rows still makes operands)
    for (int n = 0; n < rounds; ++n) {
        if (n) __syncthreads();              // everybody has read the round before
        const int own = begin + kStep * (kManyWaves * n + wave);
        if (own < end) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (own + kStep > seq.tokens || !there[h]) raw[h].vp = only_there(raw[h].vp, there[h], own + 16 * h, seq.tokens);
#pragma unroll
                for (int g = 0; g < 4; ++g) keys[2 * wave + h][g][lane] = __builtin_bit_cast(u32x4, key_operand<BITS_K>(raw[h].k, g));
                if (lane < param_words) params[2 * wave + h][lane] = param[h];
                if (lane == 0) present[2 * wave + h] = there[h];
            }
            value_operands<BITS_V>(raw, [&](int ch, half8 v0, half8 v1) {
                values[wave][ch][lane] = __builtin_bit_cast(u32x4, v0);
                values[wave][ch + 1][lane] = __builtin_bit_cast(u32x4, v1);
            });
        }
        if (n + 1 < rounds) load(n + 1);
        __syncthreads();
#pragma unroll 1
        for (int k = 0; k < kManyWaves; ++k) {
            const int token = begin + kStep * (kManyWaves * n + k);
            if (token >= end || !busy) break;
            float score[2][8];
            half8 key[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int g = 0; g < 4; ++g) key[h][g] = __builtin_bit_cast(half8, keys[2 * k + h][g][lane]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x2 ks[groups];
#pragma unroll
                for (int g = 0; g < groups; ++g) ks[g] = *(const u32x2 *)&params[2 * k + h][(q * groups + g) * 2];
                half4 zeros;
                if constexpr (groups == 4) zeros = __builtin_bit_cast(half4, *(const u32x2 *)&params[2 * k + h][32 + 2 * i]);
                else if constexpr (groups == 2) zeros = __builtin_bit_cast(half4, u32x2{params[2 * k + h][16 + i], 0u});
                else zeros = __builtin_bit_cast(half4, u32x2{(params[2 * k + h][8 + (i >> 1)] >> (16 * (i & 1))) & 0xffffu, 0u});
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    Products<GROUP> products;
                    products.make(key[h], zeros, query[t]);
                    products.scores(ks, score[t] + 4 * h);
                }
            }
            const bool have[2] = {__builtin_amdgcn_readfirstlane(present[2 * k]) != 0, __builtin_amdgcn_readfirstlane(present[2 * k + 1]) != 0};
            if (token + kStep > past || token + kStep > end || !have[0] || !have[1]) {
#pragma unroll
                for (int t = 0; t < 2; ++t) only_seen(score[t], c, seq, query[t].draft, token, past, end, have);
            }
            // values are requested before the weights are made, as many as the registers hold (when measured: 512 new tokens behind 32k, one / 8:
            // 700 / 687 us; rotated, trees of 64 over 8k, one / 4 / 8: 315 / 293 / 324)
            constexpr int early = ROTATE ? 4 : 8;
            half8 weight[2][PARTS], value[early];
#pragma unroll
            for (int ch = 0; ch < early; ++ch) value[ch] = __builtin_bit_cast(half8, values[k][ch][lane]);
            __builtin_amdgcn_s_setprio(0);
#pragma unroll
            for (int t = 0; t < 2; ++t) state[t].weigh(score[t], query[t].factor, weight[t]);
            // (a wave that has products to start goes before one with weights to make: 301 -> 293 us for trees of 64 over 8k, 718 -> 687 for 512
            // new tokens behind 32k)
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int ch = 0; ch < 8; ++ch) {
                const half8 v = ch < early ? value[ch] : __builtin_bit_cast(half8, values[k][ch][lane]);
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int t = 0; t < 2; ++t) state[t].add(ch, v, weight[t][p]);
            }
        }
    }

    constexpr int dtype = PARTS == 2 ? DT_F16 : DT_BF16;
    const int here = rows - first < kWideRows ? rows - first : kWideRows;
    const Results results{a, seq, head, first};
    if (count == 1) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float total = state[t].total(lost[32 * wave + 16 * t + i] != 0);
            const int row = 32 * wave + 16 * t + i;
            if (row < here) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x[8];
#pragma unroll
                    for (int ch = 0; ch < 8; ++ch) x[ch] = state[t].out[ch][e];
                    results.octet<dtype>(row, 32 * q + 8 * e, x, q == 0 && e == 0, state[t].top, total);
                }
            }
        }
        return;
    }
    // through LDS, where the wave has a place for 16 rows in what the keys and values had, into whole rows per 64 pairs
    const long long slot = ((long long)(part.slot0 + part.index) * each + rest) * kWideRows;
    float(*space)[kDim + 4] = (float(*)[kDim + 4]) lds;
    float(*own_rows)[kDim + 4] = space + 16 * wave;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const float total = state[t].total(lost[32 * wave + 16 * t + i] != 0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4 v;
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) v[ch] = state[t].out[4 * half + ch][e];
                *(f32x4 *)&own_rows[i][32 * q + 8 * e + 4 * half] = v;
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
        const int row0 = 32 * wave + 16 * t;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const f32x2_t v = *(const f32x2_t *)&own_rows[r][2 * lane];
            if (row0 + r < here) leave(a.part + (slot + row0 + r) * kDim + 2 * lane, v[0], v[1]);
        }
        if (q == 0 && row0 + i < here) leave(a.part_ml + 2 * (slot + row0 + i), state[t].top, total);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    }
    const unsigned first_slot = (unsigned)(part.slot0 * each + rest) * kWideRows;
    if (!last_to_arrive(a.counters + (long long)part.slot0 * each + rest, count)) return;
    const LeftRows sums_left(a.part, a.part_rows * kDim), ml_left(a.part_ml, a.part_rows * 2);
    const unsigned stride = (unsigned)each * kWideRows;
    const auto done = [&](int r, int lane_of, const float x[8], float highest, float total) {
        results.octet<dtype>(r, 8 * lane_of, x, lane_of == 0, highest, total);
    };
    if (count <= 2) join_few_parts<64 * kManyWaves, 8>(sums_left, ml_left, first_slot, stride, here, count, done);
    else if (count <= 4) join_few_parts<64 * kManyWaves, 4>(sums_left, ml_left, first_slot, stride, here, count, done);
    else if (count <= 8) join_few_parts<64 * kManyWaves, 2>(sums_left, ml_left, first_slot, stride, here, count, done);
    else join_parts<64 * kManyWaves>(sums_left, ml_left, first_slot, stride, here, count, space, done);
}

// ---- launches ---------------------------------------------------------------------------------------

template <int GROUP, bool ROTATE, int PARTS> static void launch_rows(const AttendArgs &a, int tiles, const dim3 &grid, hipStream_t stream)
{
    constexpr int bits_k = KVC_BITS / 10, bits_v = KVC_BITS % 10;
    const dim3 many(64 * kManyWaves);
    if (tiles == 1) hipLaunchKernelGGL((attend_kernel<bits_k, bits_v, GROUP, 1, ROTATE, PARTS>), grid, dim3(64 * few_waves(1, ROTATE)), 0, stream, a);
    else if (tiles == 2) hipLaunchKernelGGL((attend_kernel<bits_k, bits_v, GROUP, 2, ROTATE, PARTS>), grid, dim3(64 * few_waves(2, ROTATE)), 0, stream, a);
    else hipLaunchKernelGGL((attend_wide_kernel<bits_k, bits_v, GROUP, ROTATE, PARTS>), grid, many, 0, stream, a);
}

// fp16 results take weights in two parts, for bf16 ones (three bits less) one is enough
template <int GROUP> static void launch_group(const AttendArgs &a, int tiles, int places, hipStream_t stream)
{
    const dim3 grid((unsigned)places);
    if (a.dtype == DT_F16) {
        if (a.rotate) launch_rows<GROUP, true, 2>(a, tiles, grid, stream);
        else launch_rows<GROUP, false, 2>(a, tiles, grid, stream);
    } else {
        if (a.rotate) launch_rows<GROUP, true, 1>(a, tiles, grid, stream);
        else launch_rows<GROUP, false, 1>(a, tiles, grid, stream);
    }
}

template <> void launch_attend<KVC_BITS>(const CacheTypes &t, const AttendArgs &a, int tiles, int places, hipStream_t stream)
{
    if (t.group == 32) launch_group<32>(a, tiles, places, stream);
    else if (t.group == 64) launch_group<64>(a, tiles, places, stream);
    else launch_group<128>(a, tiles, places, stream);
}

}  // namespace kvc
