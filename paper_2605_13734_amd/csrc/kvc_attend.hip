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

// What a lane loads of one granule.
template <int BITS_K, int BITS_V, int GROUP> struct RawGranule {
    static constexpr int groups = kDim / GROUP;
    u32x4 k[BITS_K / 4], v[BITS_V / 4], vp;
    u32x2 ks[groups];                        // scales of 4 tokens
    uint32_t kz[(groups + 1) / 2];           // zeros of one token

    __device__ __forceinline__ void load(const uint8_t *p)
    {
        constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
        const int lane = lane_id(), q = lane >> 4, i = lane & 15;
#pragma unroll
        for (int h = 0; h < BITS_K / 4; ++h) k[h] = *(const u32x4 *)(p + h * 1024 + i * 64 + q * 16);
#pragma unroll
        for (int g = 0; g < groups; ++g) ks[g] = *(const u32x2 *)(p + map.k_scales + q * groups * 8 + g * 8);
        if constexpr (groups == 4) {
            const u32x2 z = *(const u32x2 *)(p + map.k_zeros + i * 8);
            kz[0] = z[0];
            kz[1] = z[1];
        } else if constexpr (groups == 2) kz[0] = *(const uint32_t *)(p + map.k_zeros + i * 4);
        else kz[0] = *(const uint16_t *)(p + map.k_zeros + i * 2);
#pragma unroll
        for (int h = 0; h < BITS_V / 4; ++h) v[h] = *(const u32x4 *)(p + map.v_codes + h * 1024 + lane * 16);
        vp = *(const u32x4 *)(p + map.v_params + (q * groups + i / (GROUP / 8)) * 16);
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

template <int BITS_K, int BITS_V, int GROUP, int TILES, bool ROTATE>
__global__ __launch_bounds__(64 * kWaves, TILES == 1 ? 2 : 1) void attend_kernel(AttendArgs a)
{
    constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
    constexpr int groups = kDim / GROUP, parts = ROTATE ? 2 : 1;
    typedef RawGranule<BITS_K, BITS_V, GROUP> Raw;
    __shared__ __attribute__((aligned(16))) float sums[kWaves][16][kDim + 4];
    __shared__ float tops[kWaves][16 * TILES], norms[kWaves][16 * TILES];

    const CacheView &c = a.c;
    const int s = blockIdx.z, head = blockIdx.y % c.heads, block = blockIdx.y / c.heads;
    const int lane = lane_id(), wave = wave_id(), q = lane >> 4, i = lane & 15;
    const Sequence seq = sequence_of(c, s);
    const int first = block * 16 * TILES, rows = seq.fresh * a.per_kv;
    if (first >= rows) return;
    const int limit = tokens_seen(c, seq, block, 16 * TILES, a.per_kv), past = seq.tokens - seq.fresh;
    const int begin = blockIdx.x * a.chunk;
    if (begin >= limit && blockIdx.x > 0) return;
    const int end = (long long)begin + a.chunk < limit ? begin + a.chunk : limit;

    // overflow of half-precision arithmetic ends at 65504 instead of infinity (bit 23 of the mode register)
    __builtin_amdgcn_s_setreg((0 << 11) | (23 << 6) | 1, 1);

    // ---- queries: column i of every tile, channels 32 g + 8 q ... of every block g
    half8 query[TILES][4 * parts];
    half4 query_sums[TILES];
    float factor[TILES];                     // scores in base 2 = (products) * factor
    int draft[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const int row = first + 16 * t + i;
        draft[t] = row < rows ? row / a.per_kv : 0;
        float x[4][8];
        const uint16_t *from = a.q + (long long)(seq.row0 + draft[t]) * a.q_row + (long long)(head * a.per_kv + row % a.per_kv) * a.q_head + 8 * q;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            u32x4 r = {0, 0, 0, 0};
            if (row < rows) r = *(const u32x4 *)(from + 32 * g);
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
        const float down = __uint_as_float((uint32_t)(127 + 7 - power) << 23);
        factor[t] = a.scale * __uint_as_float((uint32_t)(127 + power - 7) << 23) * (ROTATE ? 0.0625f : 1.0f);
        float sum[4] = {0, 0, 0, 0};
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = x[g][e] * down;
                sum[g * groups / 4] += y[e];
            }
            // the order in which unpack8 leaves the codes, 2^-20 instead of 2^-24 in every other pair at 4 bits
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int pair = e >> 1, from_e = pair + 4 * (e & 1);
                const float z = BITS_K == 4 && (pair & 1) ? y[from_e] * 0.0625f : y[from_e];
                const _Float16 high = (_Float16)z;
                query[t][g][e] = high;
                if (ROTATE) query[t][4 * (parts - 1) + g][e] = (_Float16)(z - (float)high);
            }
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float total = row_sum(sum[g]);
            const _Float16 high = (_Float16)total;
            // column i of a 16 x 16 x 16 product: lanes of q = 0 hold the sums, of q = 1 what their rounding left
            const float low = total - (float)high;
            query_sums[t][g] = g >= groups ? (_Float16)0.0f : q == 0 ? high : q == 1 ? (_Float16)low : (_Float16)0.0f;
        }
    }

    float top[TILES], norm[TILES];
    f32x4 out[TILES][8];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        top[t] = kLowest;
        norm[t] = 0.0f;
#pragma unroll
        for (int ch = 0; ch < 8; ++ch) out[t][ch] = f32x4{0, 0, 0, 0};
    }

    // ---- tokens: the wave's step n is 32 tokens from begin + 32 * (4 n + wave)
    const int steps = (end - begin + kStep - 1) / kStep;
    const int mine = steps > wave ? (steps - wave + kWaves - 1) / kWaves : 0;
    const int last_granule = (end - 1) >> 4;
    int entries = 0, ahead = -32;            // lane l: the page of granule l & 1 of the wave's step ahead + (l >> 1)
    auto load = [&](Raw *r, bool *there, int n) {
        if (n == ahead + 32) {
            ahead = n;
            const int j = (begin >> 4) + 2 * (kWaves * (n + (lane >> 1)) + wave) + (lane & 1);
            entries = page_of(c, s, j < last_granule ? j : last_granule);
            if (entries < 0) atomicOr(c.status + s, KVC_DEV_BAD_BLOCK);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = (begin >> 4) + 2 * (kWaves * n + wave) + h;
            const int page = __builtin_amdgcn_readlane(entries, 2 * (n - ahead) + h);
            there[h] = page >= 0;
            // (a granule behind the end: the last one's page, and its own place in it, which the page has)
            r[h].load(c.pages + granule_at(c, page < 0 ? 0 : page, j, head, map.bytes));
        }
    };
    auto step = [&](Raw *r, const bool *there, int n) {
        const int token = begin + kStep * (kWaves * n + wave);
        const bool plain = token + kStep <= past && token + kStep <= end && there[0] && there[1];
        if (!plain) {                        // what lies behind the end may be anything: values of zero there
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t keep[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) keep[e] = there[h] && token + 16 * h + 4 * q + e < seq.tokens ? 0xffffu : 0u;
                const uint32_t low = keep[0] | keep[1] << 16, high = keep[2] | keep[3] << 16;
                r[h].vp = u32x4{r[h].vp[0] & low, r[h].vp[1] & high, r[h].vp[2] & low, r[h].vp[3] & high};
            }
        }
        float score[TILES][8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            half8 key[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) key[g] = key_operand<BITS_K>(r[h].k, g);
            half4 zeros;
            if constexpr (groups == 4) zeros = __builtin_bit_cast(half4, u32x2{r[h].kz[0], r[h].kz[1]});
            else zeros = __builtin_bit_cast(half4, u32x2{r[h].kz[0], 0u});
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                f32x4 dot[groups];
#pragma unroll
                for (int g = 0; g < groups; ++g) dot[g] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int p = 0; p < parts; ++p)
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        dot[g * groups / 4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key[g], query[t][4 * p + g], dot[g * groups / 4], 0, 0, 0);
                const f32x4 offset = __builtin_amdgcn_mfma_f32_16x16x16f16(zeros, query_sums[t], f32x4{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float sum = 0.0f;
#pragma unroll
                    for (int g = 0; g < groups; ++g) {
                        const float scale = (float)__builtin_bit_cast(half2v, (uint32_t)r[h].ks[g][e >> 1])[e & 1];
                        sum = g ? __builtin_fmaf(scale, dot[g][e], sum) : scale * dot[g][e];
                    }
                    score[t][4 * h + e] = __builtin_fmaf(sum, 16777216.0f, offset[e]) * factor[t];
                }
            }
        }
        half8 weight[TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            if (!plain) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = token + 16 * (e >> 2) + 4 * q + (e & 3);
                    bool seen = there[e >> 2] && at < end;
                    if (seen && at >= past) seen = sees(c, seq, draft[t], at - past);
                    score[t][e] = seen ? score[t][e] : -__builtin_inff();
                }
            }
            float most = kLowest;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, score[t][e]);
            most = row_max(most);
            if (__any(most > top[t] + kSlack)) {
                const float next = fmaxf(most, top[t]), shrink = __builtin_amdgcn_exp2f(top[t] - next);
                top[t] = next;
                norm[t] *= shrink;
#pragma unroll
                for (int ch = 0; ch < 8; ++ch) out[t][ch] *= shrink;
            }
            const float down = kBias - top[t];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = __builtin_amdgcn_exp2f(score[t][e] + down);
                norm[t] += w;
                weight[t][e] = (_Float16)w;
            }
        }
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
#pragma unroll
                    for (int t = 0; t < TILES; ++t)
                        out[t][ch] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, w), weight[t], out[t][ch], 0, 0, 0);
                }
            }
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
        norm[t] = row_sum(norm[t]);
        if (q == 0) {
            tops[wave][16 * t + i] = top[t];
            norms[wave][16 * t + i] = norm[t];
        }
    }
    __syncthreads();
    const int q_heads = c.heads * a.per_kv;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        float most = kLowest;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, tops[w][16 * t + i]);
        const float share = __builtin_amdgcn_exp2f(top[t] - most);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4 v;
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) v[ch] = out[t][4 * half + ch][e] * share;
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
                *(u32x4 *)to = a.dtype == DT_F16 ? pack_row<DT_F16>(x) : pack_row<DT_BF16>(x);
                if (a.lse && i == 0)
                    a.lse[(long long)(seq.row0 + d) * q_heads + query_head] =
                        total > 0.0f ? (highest - kBias + __builtin_log2f(total)) * 0.69314718055994531f : -__builtin_inff();
            } else {
                const long long at = (((long long)s * c.max_new + d) * q_heads + query_head) * a.splits + blockIdx.x;
                *(f32x4 *)(a.part + at * kDim + 8 * i) = f32x4{x[0], x[1], x[2], x[3]};
                *(f32x4 *)(a.part + at * kDim + 8 * i + 4) = f32x4{x[4], x[5], x[6], x[7]};
                if (i == 0) *(f32x2_t *)(a.part_ml + 2 * at) = f32x2_t{highest, total};
            }
        }
        if (t + 1 < TILES) __syncthreads();
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
    if (a.lse && lane == 0)
        a.lse[(long long)(seq.row0 + d) * q_heads + query_head] =
            total > 0.0f ? (highest - kBias + __builtin_log2f(total)) * 0.69314718055994531f : -__builtin_inff();
}

// ---- launches ---------------------------------------------------------------------------------------

template <int GROUP, int TILES> static void launch_tiles(const AttendArgs &a, bool rotate, int n, hipStream_t stream)
{
    constexpr int bits_k = KVC_BITS / 10, bits_v = KVC_BITS % 10;
    const dim3 grid((unsigned)a.splits, (unsigned)(a.c.heads * a.row_blocks), (unsigned)n);
    if (rotate) hipLaunchKernelGGL((attend_kernel<bits_k, bits_v, GROUP, TILES, true>), grid, dim3(64 * kWaves), 0, stream, a);
    else hipLaunchKernelGGL((attend_kernel<bits_k, bits_v, GROUP, TILES, false>), grid, dim3(64 * kWaves), 0, stream, a);
}

template <int GROUP> static void launch_group(const AttendArgs &a, bool rotate, int tiles, int n, hipStream_t stream)
{
    if (tiles == 1) launch_tiles<GROUP, 1>(a, rotate, n, stream);
    else if (tiles == 2) launch_tiles<GROUP, 2>(a, rotate, n, stream);
    else launch_tiles<GROUP, 4>(a, rotate, n, stream);
}

template <> void launch_attend<KVC_BITS>(const CacheTypes &t, const AttendArgs &a, int tiles, int n, hipStream_t stream)
{
    if (t.group == 32) launch_group<32>(a, t.rotate, tiles, n, stream);
    else if (t.group == 64) launch_group<64>(a, t.rotate, tiles, n, stream);
    else launch_group<128>(a, t.rotate, tiles, n, stream);
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
