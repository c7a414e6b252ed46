// Attention over the quantised cache: o = sum_t softmax_t(scale * q . k_t) v_t for the new tokens of every sequence.
//
// Compiled once per pair of code widths (KVC_BITS = 10 * bits_k + bits_v).
//
// A workgroup has 16 * TILES query rows of one KV head (a row: one new token and one of the query heads that share the KV head)
// and a run of the sequence's tokens, of which its four waves take 32 at a time in turn; the waves' results are joined in
// LDS.  Where rows are few the tokens of a sequence are spread over several workgroups, whose results a second kernel joins.
//
// Scores: the matrix product runs over the codes themselves, with 16 tokens as rows and 16 query rows as columns.  A code, masked
// out of its word together with a second one, is a half-precision subnormal, code * 2^-24 (or 2^-20), which the matrix
// instructions take as it is; the group's scale multiplies the product in 32 bits and the zero enters through one more product, of
// the zeros with the sums of the query's groups: sum_d q_d (code_d scale + zero) = scale sum_d q_d code_d + zero sum_d q_d.
// So a key costs a mask per two codes and no rounding.  Queries are scaled by a power of two to a maximum in [2^7, 2^8) (exact, and
// the sums stay in the half type's range); a rotated query is the sum of two half-precision parts.
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
constexpr int kWaves = 4;
constexpr float kSlack = 8.0f;               // the maximum may grow by 2^8 before the sums are rescaled
constexpr float kBias = 6.0f;                // weights are kept as 2^(6 + score - maximum) <= 2^14
// A score that is not seen is kLowest before the factor, which is kept at 2^-60 or more (products stay below 2^40: scores below 2^-20
// instead of smaller ones), so it ends below -2^67 and weighs nothing beside the maximum that a row starts with.  A row whose scores
// are all below -2^60 counts as one that sees nothing.
constexpr float kLeastFactor = 0x1p-60f, kNothing = -0x1p60f;
constexpr float kLowest = -3.4028235e38f;

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

    __device__ __forceinline__ void load_codes(const uint8_t *p, const LanePlaces<BITS_K, BITS_V, GROUP> &at)
    {
#pragma unroll
        for (int h = 0; h < BITS_K / 4; ++h) k[h] = *(const u32x4 *)(p + at.k + h * 1024u);
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

// Channel 8 i + c of tokens t0, t1 (the words of their octets): code * scale + zero in both halves.
template <int BITS> __device__ __forceinline__ uint32_t value_pair(uint32_t pair, int c, half2v scale, half2v zero)
{
    uint32_t bits;
    _Float16 offset;
    if (BITS == 4 && (c & 1)) {
        bits = (pair & 0x00f000f0u) | 0x54005400u;            // 64 + code
        offset = (_Float16)64.0f;
    } else {
        bits = (BITS == 4 ? pair & 0x000f000fu : pair) | 0x64006400u;       // 1024 + code
        offset = (_Float16)1024.0f;
    }
    const half2v code = __builtin_bit_cast(half2v, bits) - half2v{offset, offset};
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(code, scale, zero));
}

// log of the sum of exp(scores), from the maximum in base 2 and the sum of weights
__device__ __forceinline__ float lse_of(float top, float total)
{
    return total > 0.0f ? (top - kBias + __builtin_log2f(total)) * 0.69314718055994531f : -__builtin_inff();
}

// Which of the new tokens one sees: its mask's bits, or itself and those before it.
__device__ __forceinline__ bool sees(const CacheView &c, const Sequence &seq, int draft, int j)
{
    if (c.mask == nullptr) return j <= draft;
    const unsigned long long word = c.mask[(long long)(seq.row0 + draft) * c.mask_words + (j >> 6)];
    return (word >> (j & 63)) & 1;
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

    __device__ __forceinline__ void load(const AttendArgs &a, const Sequence &seq, int head, int row, int rows)
    {
        constexpr int groups = kDim / GROUP;
        const int lane = lane_id(), q = lane >> 4;
        const bool there = row < rows;
        draft = there ? row / a.per_kv : 0;
        const uint16_t *from = a.q + (long long)(seq.row0 + draft) * a.q_row + (long long)(head * a.per_kv + row % a.per_kv) * a.q_head + 8 * q;
        float x[4][8];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            u32x4 r = {0, 0, 0, 0};
            if (there) r = *(const u32x4 *)(from + 32 * g);
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
        power = top == 0.0f ? 7 : power < -100 ? -100 : power > 119 ? 119 : power;
        float down = __uint_as_float((uint32_t)(127 + 7 - power) << 23);
        factor = fabsf(a.scale) * __uint_as_float((uint32_t)(127 + power - 7) << 23) * (ROTATE ? 0.0625f : 1.0f);
        factor = fmaxf(factor, kLeastFactor);
        if (a.scale < 0.0f) down = -down;
        float sum[4] = {0, 0, 0, 0};
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
            const _Float16 high = (_Float16)total;
            // column i of a 16 x 16 x 16 product: lanes of q = 0 hold the sums, of q = 1 what their rounding left
            const float low = total - (float)high;
            sums[g] = g >= groups ? (_Float16)0.0f : q == 0 ? high : q == 1 ? (_Float16)low : (_Float16)0.0f;
        }
    }
};

// Scores of one granule and tile from the codes: products per group, scales in 32 bits, zeros by one more product.
template <int GROUP, typename Query>
__device__ __forceinline__ void scores_of(const half8 key[4], half4 zeros, const u32x2 *ks, const Query &query, float score[4])
{
    constexpr int groups = kDim / GROUP;
    f32x4 dot[groups];
#pragma unroll
    for (int g = 0; g < groups; ++g) dot[g] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < Query::PARTS; ++p)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            dot[g * groups / 4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key[g], query.part[4 * p + g], dot[g * groups / 4], 0, 0, 0);
    const f32x4 offset = __builtin_amdgcn_mfma_f32_16x16x16f16(zeros, query.sums, f32x4{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float sum = 0.0f;
#pragma unroll
        for (int g = 0; g < groups; ++g) {
            const half2v scales = __builtin_bit_cast(half2v, (uint32_t)ks[g][e >> 1]);
            sum = __builtin_fmaf((float)scales[e & 1], dot[g][e], sum);      // (reads the half of the register as it is)
        }
        score[e] = __builtin_fmaf(sum, 16777216.0f, offset[e]);
    }
}

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
    __device__ __forceinline__ float total() const { return PARTS == 2 ? norm[0] : row_sum(norm[0]); }
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
        const float down = kBias - top;
        constexpr _Float16 one = (_Float16)1.0f;
        constexpr half8 ones = {one, one, one, one, one, one, one, one};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(score[e], factor, down));
            weight[0][e] = (_Float16)w;
            if (PARTS == 1) norm[0] += w;
            if (PARTS == 2) weight[PARTS - 1][e] = (_Float16)__builtin_fmaf((float)weight[0][e], -1.0f, w);
        }
        if (PARTS == 1) return;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) norm = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, weight[p], norm, 0, 0, 0);
    }
    __device__ __forceinline__ void add(int ch, half8 values, const half8 weight[PARTS])
    {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) out[ch] = __builtin_amdgcn_mfma_f32_16x16x32_f16(values, weight[p], out[ch], 0, 0, 0);
    }
};

// Scores of what a row does not see, of the 32 tokens from `token` on, become the lowest number.
__device__ __forceinline__ void only_seen(float score[8], const CacheView &c, const Sequence &seq, int draft, int token, int past, int end,
                                          const bool there[2])
{
    const int q = lane_id() >> 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int at = token + 16 * (e >> 2) + 4 * q + (e & 3);
        bool seen = there[e >> 2] && at < end;
        if (seen && at >= past) seen = sees(c, seq, draft, at - past);
        score[e] = seen ? score[e] : kLowest;
    }
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

// Operands of the product over tokens for channels 8 i + ch, ch = 0..7, one after the other: f(ch, operand).
template <int BITS_V, typename Raw, typename F> __device__ __forceinline__ void value_operands(const Raw *r, F f)
{
#pragma unroll
    for (int half = 0; half < BITS_V / 4; ++half)
#pragma unroll
        for (int byte = 0; byte < 4; ++byte) {
            uint32_t pair[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                pair[e] = __builtin_amdgcn_perm(r[e >> 1].v[half][2 * (e & 1) + 1], r[e >> 1].v[half][2 * (e & 1)],
                                                0x0c040c00u + (uint32_t)byte * 0x00010001u);
#pragma unroll
            for (int nibble = 0; nibble < 8 / BITS_V; ++nibble) {
                const int ch = BITS_V == 4 ? 2 * byte + nibble : 4 * half + byte;
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[e] = value_pair<BITS_V>(pair[e], ch, __builtin_bit_cast(half2v, (uint32_t)r[e >> 1].vp[e & 1]),
                                              __builtin_bit_cast(half2v, (uint32_t)r[e >> 1].vp[2 + (e & 1)]));
                f(ch, __builtin_bit_cast(half8, w));
            }
        }
}

// Pages of a wave's coming steps of 32 tokens: step n is granules first + 2 (kWaves n + wave) and the one behind it.
struct PageWindow {
    int entries, ahead;                      // lane l: the page of granule l & 1 of step ahead + (l >> 1)

    __device__ __forceinline__ void start() { ahead = -32; }
    // granule h of step n; n goes up by one from call to call (both granules of a step)
    __device__ __forceinline__ int page(const CacheView &c, int s, int first, int wave, int last, int n, int h)
    {
        if (n == ahead + 32) {
            ahead = n;
            const int lane = lane_id(), j = first + 2 * (kWaves * (n + (lane >> 1)) + wave) + (lane & 1);
            entries = page_of(c, s, j < last ? j : last);        // (behind the end: the last one's page, and a place in it)
            if (entries < 0) atomicOr(c.status + s, KVC_DEV_BAD_BLOCK);
        }
        return __builtin_amdgcn_readlane(entries, 2 * (n - ahead) + h);
    }
};

// ---- few rows: the waves of a workgroup share rows and divide tokens --------------------------------

template <int BITS_K, int BITS_V, int GROUP, int TILES, bool ROTATE, int PARTS>
__global__ __launch_bounds__(64 * kWaves, TILES == 1 ? 2 : 1) void attend_kernel(AttendArgs a)
{
    constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
    typedef RawGranule<BITS_K, BITS_V, GROUP> Raw;
    __shared__ __attribute__((aligned(16))) float sums[kWaves][16][kDim + 4];
    __shared__ float tops[kWaves][16 * TILES], norms[kWaves][16 * TILES];

    const CacheView &c = a.c;
    const int s = blockIdx.z, split = (int)(blockIdx.x % (unsigned)a.splits), place = (int)(blockIdx.x / (unsigned)a.splits);
    const int head = place % c.heads, block = place / c.heads;
    const int lane = lane_id(), wave = wave_id(), q = lane >> 4, i = lane & 15;
    const Sequence seq = sequence_of(c, s);
    const int first = block * 16 * TILES, rows = seq.fresh * a.per_kv;
    if (first >= rows) return;
    const int limit = tokens_seen(c, seq, block, 16 * TILES, a.per_kv), past = seq.tokens - seq.fresh;
    const long long start = (long long)split * a.chunk;
    if (start >= limit) return;
    const int begin = (int)start;
    const int end = start + a.chunk < limit ? begin + a.chunk : limit;

    // overflow of half-precision arithmetic ends at 65504 instead of infinity (bit 23 of the mode register)
    __builtin_amdgcn_s_setreg((0 << 11) | (23 << 6) | 1, 1);

    QueryTile<BITS_K, GROUP, ROTATE> query[TILES];
    RowState<PARTS> state[TILES];
    LanePlaces<BITS_K, BITS_V, GROUP> at;
    at.set();
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        query[t].load(a, seq, head, first + 16 * t + i, rows);
        state[t].clear();
    }

    // ---- tokens: the wave's step n is 32 tokens from begin + 32 * (4 n + wave)
    const int steps = (end - begin + kStep - 1) / kStep;
    const int mine = steps > wave ? (steps - wave + kWaves - 1) / kWaves : 0;
    PageWindow window;
    window.start();
    auto load = [&](Raw *r, bool *there, int n) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int page = window.page(c, s, begin >> 4, wave, (end - 1) >> 4, n, h);
            there[h] = page >= 0;
            const uint8_t *p = c.pages + granule_at(c, page < 0 ? 0 : page, (begin >> 4) + 2 * (kWaves * n + wave) + h, head, map.bytes);
            r[h].load_codes(p, at);
            r[h].load_scales(p, at);
        }
    };
    auto step = [&](Raw *r, const bool *there, int n) {
        const int token = begin + kStep * (kWaves * n + wave);
        const bool all = token + kStep <= past && token + kStep <= end && there[0] && there[1];
        if (!all) {
#pragma unroll
            for (int h = 0; h < 2; ++h) r[h].vp = only_there(r[h].vp, there[h], token + 16 * h, seq.tokens);
        }
        float score[TILES][8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            half8 key[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) key[g] = key_operand<BITS_K>(r[h].k, g);
#pragma unroll
            for (int t = 0; t < TILES; ++t) scores_of<GROUP>(key, r[h].zeros(), r[h].ks, query[t], score[t] + 4 * h);
        }
        if (!all) {
#pragma unroll
            for (int t = 0; t < TILES; ++t) only_seen(score[t], c, seq, query[t].draft, token, past, end, there);
        }
        half8 weight[TILES][PARTS];
#pragma unroll
        for (int t = 0; t < TILES; ++t) state[t].weigh(score[t], query[t].factor, weight[t]);
        value_operands<BITS_V>(r, [&](int ch, half8 values) {
#pragma unroll
            for (int t = 0; t < TILES; ++t) state[t].add(ch, values, weight[t]);
        });
    };
    Raw now[2], next[2];
    bool now_there[2] = {false, false}, next_there[2] = {false, false};
    if (mine > 0) load(now, now_there, 0);
    for (int n = 0; n < mine; n += 2) {
        if (n + 1 < mine) load(next, next_there, n + 1);
        step(now, now_there, n);
        if (n + 1 < mine) {
            if (n + 2 < mine) load(now, now_there, n + 2);
            step(next, next_there, n + 1);
        }
    }

    // ---- the waves' results: maxima and sums first, then the rows, a tile at a time
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const float total = state[t].total();
        if (q == 0) {
            tops[wave][16 * t + i] = state[t].top;
            norms[wave][16 * t + i] = total;
        }
    }
    __syncthreads();
    const int q_heads = c.heads * a.per_kv;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        float most = kLowest;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, tops[w][16 * t + i]);
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
        // the wave finishes rows 4 * wave + q, 8 channels per lane
        const int r = 4 * wave + q, row = first + 16 * t + r;
        if (row < rows) {
            float x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, total = 0.0f, highest = kLowest;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) highest = fmaxf(highest, tops[w][16 * t + r]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                total += norms[w][16 * t + r] * __builtin_amdgcn_exp2f(tops[w][16 * t + r] - highest);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] += sums[w][r][8 * i + e];
            }
            const int d = row / a.per_kv, query_head = head * a.per_kv + row % a.per_kv;
            if (a.splits == 1) {
                const float part = total > 0.0f ? 1.0f / total : 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= part;
                uint16_t *to = a.out + (long long)(seq.row0 + d) * a.o_row + (long long)query_head * a.o_head + 8 * i;
                *(u32x4 *)to = PARTS == 2 ? pack_row<DT_F16>(x) : pack_row<DT_BF16>(x);
                if (a.lse && i == 0) a.lse[(long long)(seq.row0 + d) * q_heads + query_head] = lse_of(highest, total);
            } else {
                const long long at = (((long long)s * c.max_new + d) * q_heads + query_head) * a.splits + split;
                *(f32x4 *)(a.part + at * kDim + 8 * i) = f32x4{x[0], x[1], x[2], x[3]};
                *(f32x4 *)(a.part + at * kDim + 8 * i + 4) = f32x4{x[4], x[5], x[6], x[7]};
                if (i == 0) *(f32x2_t *)(a.part_ml + 2 * at) = f32x2_t{highest, total};
            }
        }
        if (t + 1 < TILES) __syncthreads();
    }
}

// ---- many rows: the waves of a workgroup share tokens and divide rows --------------------------------

// 128 tokens at a time: each wave turns 32 of them into operands, which go through LDS in the order of the lanes (every access is
// one KB in a row); each wave has 32 rows.
template <int BITS_K, int BITS_V, int GROUP, bool ROTATE, int PARTS>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_wide_kernel(AttendArgs a)
{
    constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
    constexpr int groups = kDim / GROUP, param_words = 16 * groups;      // words of a granule's key scales and zeros
    typedef RawGranule<BITS_K, BITS_V, GROUP> Raw;
    __shared__ u32x4 keys[2 * kWaves][4][64], values[kWaves][8][64];
    __shared__ __attribute__((aligned(16))) uint32_t params[2 * kWaves][param_words];
    __shared__ int present[2 * kWaves];

    const CacheView &c = a.c;
    const int s = blockIdx.z, split = (int)(blockIdx.x % (unsigned)a.splits), place = (int)(blockIdx.x / (unsigned)a.splits);
    const int head = place % c.heads, block = place / c.heads;
    const int lane = lane_id(), wave = wave_id(), q = lane >> 4, i = lane & 15;
    const Sequence seq = sequence_of(c, s);
    const int first = block * kWideRows, rows = seq.fresh * a.per_kv;
    if (first >= rows) return;
    const int limit = tokens_seen(c, seq, block, kWideRows, a.per_kv), past = seq.tokens - seq.fresh;
    const long long start = (long long)split * a.chunk;
    if (start >= limit) return;
    const int begin = (int)start;
    const int end = start + a.chunk < limit ? begin + a.chunk : limit;
    __builtin_amdgcn_s_setreg((0 << 11) | (23 << 6) | 1, 1);             // (see attend_kernel)

    QueryTile<BITS_K, GROUP, ROTATE> query[2];
    RowState<PARTS> state[2];
    LanePlaces<BITS_K, BITS_V, GROUP> at;
    at.set();
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        query[t].load(a, seq, head, first + 32 * wave + 16 * t + i, rows);
        state[t].clear();
    }

    const int steps = (end - begin + kStep - 1) / kStep, rounds = (steps + kWaves - 1) / kWaves;
    PageWindow window;
    window.start();
    Raw raw[2];
    uint32_t param[2];
    bool there[2] = {false, false};
    auto load = [&](int n) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int page = window.page(c, s, begin >> 4, wave, (end - 1) >> 4, n, h);
            there[h] = page >= 0;
            const uint8_t *p = c.pages + granule_at(c, page < 0 ? 0 : page, (begin >> 4) + 2 * (kWaves * n + wave) + h, head, map.bytes);
            raw[h].load_codes(p, at);
            param[h] = *(const uint32_t *)(p + map.k_scales + (uint32_t)(lane % param_words) * 4u);
        }
    };
    load(0);
    for (int n = 0; n < rounds; ++n) {
        if (n) __syncthreads();              // everybody has read the round before
        const int own = begin + kStep * (kWaves * n + wave);
        if (own < end) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (own + kStep > seq.tokens || !there[h]) raw[h].vp = only_there(raw[h].vp, there[h], own + 16 * h, seq.tokens);
#pragma unroll
                for (int g = 0; g < 4; ++g) keys[2 * wave + h][g][lane] = __builtin_bit_cast(u32x4, key_operand<BITS_K>(raw[h].k, g));
                if (lane < param_words) params[2 * wave + h][lane] = param[h];
                if (lane == 0) present[2 * wave + h] = there[h];
            }
            value_operands<BITS_V>(raw, [&](int ch, half8 v) { values[wave][ch][lane] = __builtin_bit_cast(u32x4, v); });
        }
        if (n + 1 < rounds) load(n + 1);
        __syncthreads();
#pragma unroll 1
        for (int k = 0; k < kWaves; ++k) {
            const int token = begin + kStep * (kWaves * n + k);
            if (token >= end) break;
            float score[2][8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                half8 key[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) key[g] = __builtin_bit_cast(half8, keys[2 * k + h][g][lane]);
                u32x2 ks[groups];
#pragma unroll
                for (int g = 0; g < groups; ++g) ks[g] = *(const u32x2 *)&params[2 * k + h][(q * groups + g) * 2];
                half4 zeros;
                if constexpr (groups == 4) zeros = __builtin_bit_cast(half4, *(const u32x2 *)&params[2 * k + h][32 + 2 * i]);
                else if constexpr (groups == 2) zeros = __builtin_bit_cast(half4, u32x2{params[2 * k + h][16 + i], 0u});
                else zeros = __builtin_bit_cast(half4, u32x2{(params[2 * k + h][8 + (i >> 1)] >> (16 * (i & 1))) & 0xffffu, 0u});
#pragma unroll
                for (int t = 0; t < 2; ++t) scores_of<GROUP>(key, zeros, ks, query[t], score[t] + 4 * h);
            }
            const bool have[2] = {__builtin_amdgcn_readfirstlane(present[2 * k]) != 0, __builtin_amdgcn_readfirstlane(present[2 * k + 1]) != 0};
            if (token + kStep > past || token + kStep > end || !have[0] || !have[1]) {
#pragma unroll
                for (int t = 0; t < 2; ++t) only_seen(score[t], c, seq, query[t].draft, token, past, end, have);
            }
            half8 weight[2][PARTS];
#pragma unroll
            for (int t = 0; t < 2; ++t) state[t].weigh(score[t], query[t].factor, weight[t]);
#pragma unroll
            for (int ch = 0; ch < 8; ++ch) {
                const half8 v = __builtin_bit_cast(half8, values[k][ch][lane]);
#pragma unroll
                for (int t = 0; t < 2; ++t) state[t].add(ch, v, weight[t]);
            }
        }
    }

    const int q_heads = c.heads * a.per_kv;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const float total = state[t].total();
        const int row = first + 32 * wave + 16 * t + i;
        if (row < rows) {
            const int d = row / a.per_kv, query_head = head * a.per_kv + row % a.per_kv;
            if (a.splits == 1) {
                const float part = total > 0.0f ? 1.0f / total : 0.0f;
                uint16_t *to = a.out + (long long)(seq.row0 + d) * a.o_row + (long long)query_head * a.o_head + 32 * q;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x[8];
#pragma unroll
                    for (int ch = 0; ch < 8; ++ch) x[ch] = state[t].out[ch][e] * part;
                    *(u32x4 *)(to + 8 * e) = PARTS == 2 ? pack_row<DT_F16>(x) : pack_row<DT_BF16>(x);
                }
                if (a.lse && q == 0) a.lse[(long long)(seq.row0 + d) * q_heads + query_head] = lse_of(state[t].top, total);
            } else {
                const long long place_of = (((long long)s * c.max_new + d) * q_heads + query_head) * a.splits + split;
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        f32x4 v;
#pragma unroll
                        for (int ch = 0; ch < 4; ++ch) v[ch] = state[t].out[4 * half + ch][e];
                        *(f32x4 *)(a.part + place_of * kDim + 32 * q + 8 * e + 4 * half) = v;
                    }
                if (q == 0) *(f32x2_t *)(a.part_ml + 2 * place_of) = f32x2_t{state[t].top, total};
            }
        }
    }
}

// Joins the splits of a query row: one wave per row, 16 lanes with 8 channels each, the splits dealt to the four sets of lanes.
template <int DT>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, int rows_per_block)
{
    const CacheView &c = a.c;
    const int s = blockIdx.z, q_heads = c.heads * a.per_kv, lane = lane_id(), q = lane >> 4, i = lane & 15;
    const Sequence seq = sequence_of(c, s);
    const int at_row = (int)blockIdx.x * 4 + wave_id(), d = at_row / q_heads, query_head = at_row % q_heads;
    if (d >= seq.fresh) return;
    const int block = (int)(((long long)d * a.per_kv + query_head % a.per_kv) / rows_per_block);
    const int splits = (tokens_seen(c, seq, block, rows_per_block, a.per_kv) + a.chunk - 1) / a.chunk;
    const long long at = (((long long)s * c.max_new + d) * q_heads + query_head) * a.splits;
    float highest = kLowest;
    for (int k = lane; k < splits; k += 64) highest = fmaxf(highest, a.part_ml[2 * (at + k)]);
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) highest = fmaxf(highest, __shfl_xor(highest, m, 64));
    highest = row_max(highest);
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, total = 0.0f;
    for (int k = q; k < splits; k += 4) {
        const f32x2_t ml = *(const f32x2_t *)(a.part_ml + 2 * (at + k));
        const f32x4 lo = *(const f32x4 *)(a.part + (at + k) * kDim + 8 * i), hi = *(const f32x4 *)(a.part + (at + k) * kDim + 8 * i + 4);
        const float share = __builtin_amdgcn_exp2f(ml[0] - highest);
        total = __builtin_fmaf(ml[1], share, total);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = __builtin_fmaf(lo[e], share, x[e]);
            x[4 + e] = __builtin_fmaf(hi[e], share, x[4 + e]);
        }
    }
    total = row_sum(total);
    const float part = total > 0.0f ? 1.0f / total : 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = row_sum(x[e]) * part;
    if (q == 0) {
        uint16_t *to = a.out + (long long)(seq.row0 + d) * a.o_row + (long long)query_head * a.o_head + 8 * i;
        *(u32x4 *)to = pack_row<DT>(x);
    }
    if (a.lse && lane == 0) a.lse[(long long)(seq.row0 + d) * q_heads + query_head] = lse_of(highest, total);
}

// ---- launches ---------------------------------------------------------------------------------------

template <int GROUP, bool ROTATE, int PARTS> static void launch_rows(const AttendArgs &a, int tiles, const dim3 &grid, hipStream_t stream)
{
    constexpr int bits_k = KVC_BITS / 10, bits_v = KVC_BITS % 10;
    const dim3 threads(64 * kWaves);
    if (tiles == 1) hipLaunchKernelGGL((attend_kernel<bits_k, bits_v, GROUP, 1, ROTATE, PARTS>), grid, threads, 0, stream, a);
    else if (tiles == 2) hipLaunchKernelGGL((attend_kernel<bits_k, bits_v, GROUP, 2, ROTATE, PARTS>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((attend_wide_kernel<bits_k, bits_v, GROUP, ROTATE, PARTS>), grid, threads, 0, stream, a);
}

// fp16 results take weights in two parts, for bf16 ones (three bits less) one is enough
template <int GROUP> static void launch_group(const AttendArgs &a, int tiles, int n, hipStream_t stream)
{
    const dim3 grid((unsigned)a.splits * (unsigned)(a.c.heads * a.row_blocks), 1, (unsigned)n);
    if (a.dtype == DT_F16) {
        if (a.rotate) launch_rows<GROUP, true, 2>(a, tiles, grid, stream);
        else launch_rows<GROUP, false, 2>(a, tiles, grid, stream);
    } else {
        if (a.rotate) launch_rows<GROUP, true, 1>(a, tiles, grid, stream);
        else launch_rows<GROUP, false, 1>(a, tiles, grid, stream);
    }
}

template <> void launch_attend<KVC_BITS>(const CacheTypes &t, const AttendArgs &a, int tiles, int n, hipStream_t stream)
{
    if (t.group == 32) launch_group<32>(a, tiles, n, stream);
    else if (t.group == 64) launch_group<64>(a, tiles, n, stream);
    else launch_group<128>(a, tiles, n, stream);
}

#if KVC_BITS == 44          // (all widths join the same way: one of the units has the kernel)
void launch_attend_join(const AttendArgs &a, int tiles, int n, hipStream_t stream)
{
    const dim3 grid((unsigned)(((long long)a.c.max_new * a.c.heads * a.per_kv + 3) / 4), 1, (unsigned)n);
    if (a.dtype == DT_F16) hipLaunchKernelGGL(attend_join_kernel<DT_F16>, grid, dim3(256), 0, stream, a, 16 * tiles);
    else hipLaunchKernelGGL(attend_join_kernel<DT_BF16>, grid, dim3(256), 0, stream, a, 16 * tiles);
}
#endif

}  // namespace kvc
