// Causal attention over whole prompts, packed one after the other: o_i = sum_{j <= i} softmax_j(scale * q_i . k_j) v_j.
//
// A workgroup has a block of rows of one query head, its waves divide the rows; tiles of 64 tokens of K and V go through LDS and are read
// by all waves.  The scores' product has the keys as rows and the queries as columns (16 x 16 x 32): a lane then holds the scores of
// one row and of the tokens 4 g ... 4 g + 3 of a tile of 16 (lane = 16 g + i, row i), two of which are, as weights, the operand that the
// second product takes for 32 tokens: nothing moves between lanes.  The values' operand holds the same tokens, read from LDS with the
// transposing load (4 tokens x 16 channels per 16 lanes).  Results stand with channels as rows and queries as columns, so a row's maximum and
// sum belong to the lanes that hold its results.
// Softmax: running maximum and sum per row in 32 bits, base 2.  Lanes look for a maximum of their own tokens only; the four lanes of a row
// meet when one of them has found a score more than 2^kSlack above the maximum that the row's weights refer to (or none was there yet).
// Weights are kept as 2^(kBias + score - maximum) <= 2^15, inside the half type, so that weights down to 2^-39 of the largest count.
//
// What a row does not see must not matter whatever it holds: scores are replaced (not added to) where tokens are behind the row, but a
// weight of zero times a value that is NaN or infinite is NaN.  That is looked for once, in the results: a block that has one that is no
// finite number is done again with the values of the tiles that some rows see and others do not taken as zero where they are
// not finite, and as NaN by the rows that see them.
#include "kvc_prompt_internal.h"
#include "../../include/kvc.h"

namespace kvc {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bhalf2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;                    // tokens of K and V in LDS
constexpr int kGroup = 32;                   // tokens of a step
constexpr float kSlack = 7.0f, kBias = 8.0f;
constexpr float kNone = -__builtin_inff();
constexpr int kSorted = 256;                 // sequences of a call whose blocks are taken longest first

template <int DT> __device__ __forceinline__ f32x4 multiply(const u32x4 &a, const u32x4 &b, f32x4 c)
{
    if constexpr (DT == DT_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), c, 0, 0, 0);
}
template <int DT> __device__ __forceinline__ uint32_t round_pair(float a, float b)
{
    const f32x2 x = {a, b};
    if constexpr (DT == DT_F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, half2v));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bhalf2));
}

// maximum and sum over the four lanes that hold one row
__device__ __forceinline__ float max_of_row(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_of_row(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ long long sum_of_wave(long long x)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m, 64);
    return x;
}

// ---- which block ------------------------------------------------------------------------------------

struct Block {
    int row0, rows;                          // of the sequence
    int first;                               // of the block, in the sequence
    long long all;                           // blocks of the call, where that is known
};

// Rows of sequence s, none where its numbers do not fit (reported).
__device__ __forceinline__ int rows_of(const PromptArgs &a, int s, int &row0)
{
    row0 = a.start[s];
    const int rows = (int)((unsigned)a.start[s + 1] - (unsigned)row0);
    if (row0 >= 0 && (unsigned)rows <= (unsigned)a.max_rows && (long long)row0 + rows <= a.rows) return rows;
    if (blockIdx.x == 0 && threadIdx.x < 64) atomicOr(a.status + s, KVC_DEV_BAD_ROW);
    return 0;
}

// Block `number` of all blocks of `size` rows, the same in all lanes; false where there are fewer.  The blocks of up to kSorted sequences
// come longest first (those with most tokens before them, over all sequences), so that the last ones to run are short; those of more
// sequences in the order of the sequences, each from its end.
__device__ __forceinline__ bool find_block(const PromptArgs &a, long long number, int size, Block &b)
{
    const int lane = lane_id();
    int at, row0;
    if (a.n <= kSorted) {
        int blocks[kSorted / 64];
        long long all = 0;
        int most = 0;
#pragma unroll
        for (int i = 0; i < kSorted / 64; ++i) {
            const int s = 64 * i + lane;
            blocks[i] = s < a.n ? (int)(((unsigned)rows_of(a, s, row0) + size - 1) / size) : 0;
            all += blocks[i];
            most = most > blocks[i] ? most : blocks[i];
        }
        if (a.n > 1) {
            all = sum_of_wave(all);
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const int x = __shfl_xor(most, m, 64);
                most = most > x ? most : x;
            }
        } else {
            all = __builtin_amdgcn_readfirstlane((int)all);
            most = (int)all;
        }
        b.all = all;
        if (number >= all) return false;
        // the highest level (blocks before it in its sequence) at and above which there are more than `number` blocks
        int low = 0, high = most;            // (low: more than `number`; high: no more)
        long long above = 0;                 // blocks at and above `high`
        if (a.n == 1) {
            low = most - 1 - (int)number;
            above = number;
        }
        while (a.n > 1 && high - low > 1) {
            const int mid = (low + high) >> 1;
            long long sum = 0;
#pragma unroll
            for (int i = 0; i < kSorted / 64; ++i) sum += blocks[i] > mid ? blocks[i] - mid : 0;
            sum = sum_of_wave(sum);
            if (sum > number) low = mid;
            else {
                high = mid;
                above = sum;
            }
        }
        // the (number - above)-th sequence that has a block at this level
        int left = (int)(number - above), s = 0;
#pragma unroll
        for (int i = 0; i < kSorted / 64; ++i) {
            unsigned long long have = __ballot(blocks[i] > low);
            const int many = __popcll(have);
            if (left >= 0 && left < many) {
                for (int k = 0; k < left; ++k) have &= have - 1;
                s = 64 * i + __ffsll((unsigned long long)have) - 1;
            }
            left -= many;
        }
        s = __builtin_amdgcn_readfirstlane(s);
        b.rows = __builtin_amdgcn_readfirstlane(rows_of(a, s, row0));
        at = low;
    } else {
        b.all = INT64_MAX / 65536;
        int s = -1, mine = 0;
        long long before = 0;
        for (int i = 0; i < a.n; i += 64) {
            mine = i + lane < a.n ? (int)(((unsigned)rows_of(a, i + lane, row0) + size - 1) / size) : 0;
            long long sum = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const long long up = __shfl_up(sum, d, 64);
                if (lane >= d) sum += up;
            }
            const unsigned long long have = __ballot(before + sum > number);
            if (have && s < 0) {
                const int l = __ffsll((unsigned long long)have) - 1;
                s = i + l;
                at = (int)(before + __shfl(sum, l, 64) - 1 - number);
                if (blockIdx.x) break;       // (the first workgroup looks at all sequences for its reports)
            }
            before += __shfl(sum, 63, 64);
        }
        if (s < 0) return false;
        s = __builtin_amdgcn_readfirstlane(s);
        at = __builtin_amdgcn_readfirstlane(at);
        b.rows = __builtin_amdgcn_readfirstlane(rows_of(a, s, row0));
    }
    b.row0 = __builtin_amdgcn_readfirstlane(row0);
    b.first = at * size;
    return true;
}

// ---- the kernel -----------------------------------------------------------------------------------

// Octet of channels c of token t of a tile, in 16-byte pieces: rows of 16 pieces, turned so that the 16 tokens that lanes read at one octet
// (keys), and the 8 tokens of which they read 32 bytes (values), lie in different banks.
__device__ __forceinline__ int key_piece(int t, int c) { return t * 16 + (c ^ (t & 15)); }
__device__ __forceinline__ int value_piece(int t, int c) { return t * 16 + (c ^ ((t & 7) << 1)); }

// Numbers that are not finite as zero; `lost` has the type's 1 in their place and 0 elsewhere.
template <int DT> __device__ __forceinline__ void only_finite(u32x4 &x, u32x4 &lost)
{
    constexpr uint32_t top = DT == DT_F16 ? 0x7c00u : 0x7f80u, one = DT == DT_F16 ? 0x3c00u : 0x3f80u;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const bool low = (x[w] & top) == top, high = ((x[w] >> 16) & top) == top;
        lost[w] = (low ? one : 0u) | (high ? one << 16 : 0u);
        x[w] &= (low ? 0u : 0xffffu) | (high ? 0u : 0xffff0000u);
    }
}

template <int DT, int TILES> __global__ __launch_bounds__(64 * kPromptWaves, 2) void prompt_kernel(PromptArgs a, long long places)
{
    constexpr int kRows = 16 * TILES, kBlock = kRows * kPromptWaves;
    __shared__ u32x4 keys[kTile * 16], values[kTile * 16];
    const int lane = lane_id(), wave = wave_id(), i = lane & 15, g = lane >> 4;
    const int q_heads = a.kv_heads * a.per_kv;
    for (long long place = blockIdx.x;; place += places) {
        // neighbouring workgroups, which run on different XCDs, have different KV heads; those of one KV head meet in an L2
        const int kv = (int)(place % a.kv_heads);
        const int head = kv * a.per_kv + (int)(place / a.kv_heads % a.per_kv);
        Block b;
        if (!find_block(a, place / q_heads, kBlock, b)) return;
        const int first = b.first + wave * kRows;                  // of the wave
        const uint16_t *q_at = a.q + (long long)b.row0 * a.q_row + head * a.q_head;
        const uint16_t *k_at = a.k + (long long)b.row0 * a.k_row + kv * a.k_head;
        const uint16_t *v_at = a.v + (long long)b.row0 * a.v_row + kv * a.v_head;
        const int tokens = b.first + kBlock < b.rows ? b.first + kBlock : b.rows;
        u32x4 query[TILES][4];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const int row = first + 16 * t + i < b.rows ? first + 16 * t + i : b.rows - 1;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                query[t][c] = *(const u32x4 *)(q_at + (long long)row * a.q_row + 32 * c + 8 * g);
                query[t][c] = (query[t][c] & a.query_and) ^ a.query_xor;
            }
        }
        f32x4 out[TILES][8];
        float top[TILES], shift[TILES], sum[TILES];
        bool again = false;
        for (;;) {
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                top[t] = kNone;
                shift[t] = kBias;
                sum[t] = 0.0f;
#pragma unroll
                for (int d = 0; d < 8; ++d) out[t][d] = f32x4{0, 0, 0, 0};
            }
            for (int at = 0; at < tokens; at += kTile) {
                __syncthreads();
#pragma unroll
                for (int r = 0; r < kTile * 16 / (64 * kPromptWaves); ++r) {
                    const int piece = r * 64 * kPromptWaves + threadIdx.x, token = piece >> 4, c = piece & 15;
                    u32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
                    if (at + token < b.rows) {
                        x = *(const u32x4 *)(k_at + (long long)(at + token) * a.k_row + 8 * c);
                        y = *(const u32x4 *)(v_at + (long long)(at + token) * a.v_row + 8 * c);
                    }
                    keys[key_piece(token, c)] = x;
                    values[value_piece(token, c)] = y;
                }
                __syncthreads();
                for (int step = 0; step < kTile; step += kGroup) {
                    const int token = at + step;
                    if (first >= b.rows || token >= first + kRows) break;
                    const bool mixed = token + kGroup - 1 > first;           // some rows see some of the tokens only
                    float score[TILES][8];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        f32x4 s[TILES];
#pragma unroll
                        for (int t = 0; t < TILES; ++t) s[t] = f32x4{0, 0, 0, 0};
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const u32x4 key = keys[key_piece(step + 16 * h + i, 4 * c + g)];
#pragma unroll
                            for (int t = 0; t < TILES; ++t) s[t] = multiply<DT>(key, query[t][c], s[t]);
                        }
#pragma unroll
                        for (int t = 0; t < TILES; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) score[t][4 * h + e] = s[t][e];
                    }
                    if (mixed) {
#pragma unroll
                        for (int t = 0; t < TILES; ++t)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (token + 16 * (e >> 2) + 4 * g + (e & 3) > first + 16 * t + i) score[t][e] = kNone;
                    }
                    bool grown = false;
                    float most[TILES];
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        most[t] = score[t][0];
#pragma unroll
                        for (int e = 1; e < 8; ++e) most[t] = fmaxf(most[t], score[t][e]);
                        grown |= __builtin_fmaf(most[t], a.factor, -top[t]) > kSlack;
                    }
                    if (__any(grown)) {
#pragma unroll
                        for (int t = 0; t < TILES; ++t) {
                            // (rows that have not grown stay as they are: a row's bits depend on what it sees alone)
                            const float highest = max_of_row(most[t]);
                            const float now = __builtin_fmaf(highest, a.factor, -top[t]) > kSlack ? highest * a.factor : top[t];
                            const float from = now == kNone ? 0.0f : now;
                            const float by = __builtin_amdgcn_exp2f(top[t] - from);
                            top[t] = now;
                            shift[t] = kBias - from;
                            sum[t] *= by;
#pragma unroll
                            for (int d = 0; d < 8; ++d) out[t][d] *= by;
                        }
                    }
                    u32x4 weight[TILES];
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        float w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(score[t][e], a.factor, shift[t]));
                            sum[t] += w[e];
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) weight[t][e] = round_pair<DT>(w[2 * e], w[2 * e + 1]);
                    }
#pragma unroll
                    for (int d = 0; d < 8; ++d) {
                        // token 4 g + i / 4 of the lane's 16 (then 16 further), channels 16 d + 4 (i % 4) ... + 3; the lane gets tokens
                        // 4 g ... 4 g + 3 of channel 16 d + i
                        u32x4 value;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int t = step + 16 * h + 4 * g + (i >> 2);
                            const char *from = (const char *)&values[value_piece(t, 2 * d + ((i & 3) >> 1))] + 8 * (i & 1);
                            const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                (__attribute__((address_space(3))) s16x4 *)from));
                            value[2 * h] = x[0];
                            value[2 * h + 1] = x[1];
                        }
                        if (mixed && again) {
                            u32x4 lost;
                            only_finite<DT>(value, lost);
#pragma unroll
                            for (int t = 0; t < TILES; ++t) {
                                u32x4 seen;
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int behind = first + 16 * t + i - (token + 16 * (e >> 1) + 4 * g + 2 * (e & 1));
                                    constexpr uint32_t one = DT == DT_F16 ? 0x3c00u : 0x3f80u;
                                    seen[e] = (behind >= 0 ? one : 0u) | (behind >= 1 ? one << 16 : 0u);
                                }
                                const f32x4 count = multiply<DT>(lost, seen, f32x4{0, 0, 0, 0});
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (count[e] > 0.0f) out[t][d][e] = __builtin_nanf("");
                            }
                        }
#pragma unroll
                        for (int t = 0; t < TILES; ++t) out[t][d] = multiply<DT>(value, weight[t], out[t][d]);
                    }
                }
            }
            bool finite = true;
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int d = 0; d < 8; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) finite &= out[t][d][e] - out[t][d][e] == 0.0f;
            finite |= first >= b.rows;
            if (again || !__syncthreads_or(!finite)) break;
            again = true;
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const int row = first + 16 * t + i;
            const float all = sum_of_row(sum[t]), by = 1.0f / all;
            if (row >= b.rows) continue;
            uint16_t *to = a.out + (long long)(b.row0 + row) * a.o_row + head * a.o_head + 4 * g;
#pragma unroll
            for (int d = 0; d < 8; ++d)
                *(u32x2 *)(to + 16 * d) = u32x2{round_pair<DT>(out[t][d][0] * by, out[t][d][1] * by), round_pair<DT>(out[t][d][2] * by, out[t][d][3] * by)};
            if (a.lse && g == 0)
                a.lse[(long long)(b.row0 + row) * q_heads + head] = (__builtin_amdgcn_logf(all) - shift[t]) * 0.693147181f;
        }
        if (place + places >= b.all * q_heads) return;
        __syncthreads();
    }
}

PromptShape prompt_shape(const PromptArgs &a)
{
    PromptShape s;
    s.tiles = 2;
    const long long size = 16 * s.tiles * kPromptWaves, each = (a.max_rows + size - 1) / size;
    // blocks of all sequences: no more than what their number and bound allow, or their rows in all
    long long blocks = each * a.n, most = a.rows / size + a.n;
    blocks = blocks < most ? blocks : most;
    s.places = blocks * a.kv_heads * a.per_kv;
    const long long limit = 1 << 22;         // (further blocks are taken in turn, which also covers starts that overlap)
    s.places = s.places < 1 ? 1 : s.places > limit ? limit : s.places;
    return s;
}

template <int DT> static void launch_type(const PromptArgs &a, const PromptShape &s, hipStream_t stream)
{
    prompt_kernel<DT, 2><<<dim3((unsigned)s.places), 64 * kPromptWaves, 0, stream>>>(a, s.places);
}
void launch_prompt(int dtype, const PromptArgs &a, const PromptShape &s, hipStream_t stream)
{
    if (dtype == DT_F16) launch_type<DT_F16>(a, s, stream);
    else launch_type<DT_BF16>(a, s, stream);
}

}  // namespace kvc
