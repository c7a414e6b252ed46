// Causal attention over whole prompts, packed one after the other: o_i = sum_{j <= i} softmax_j(scale * q_i . k_j) v_j.
//
// A workgroup has a block of rows of one query head, its waves divide the rows; tiles of 32 or 64 tokens of K and V go through LDS and are read
// by all waves.  The scores' product has the keys as rows and the queries as columns (16 x 16 x 32): a lane then holds the scores of
// one row and of the tokens 4 g ... 4 g + 3 of a tile of 16 (lane = 16 g + i, row i), two of which are, as weights, the operand that the
// second product takes for 32 tokens: nothing moves between lanes.  The values' operand holds the same tokens, read from LDS with the
// transposing load (4 tokens x 16 channels per 16 lanes).  Results stand with channels as rows and queries as columns, so a row's maximum and
// sum belong to the lanes that hold its results.
// Softmax: running maximum and sum per row in 32 bits, base 2.  Lanes look for a maximum of their own tokens only; the four lanes of a row
// meet when one of them has found a score more than 2^kSlack above the maximum that the row's weights refer to (or none was there yet).
//
// What a row does not see must not matter whatever it holds: scores are replaced (not added to) where tokens are behind the row, but a
// weight of zero times a value that is NaN or infinite is NaN.  That is looked for once, in the results: a block that has one that is no
// finite number is done again with the values of the tiles that some rows see and others do not taken as zero where they are
// not finite, and as NaN by the rows that see them.
//
// What bounds it: long prompts the matrix products beside the softmax's instructions (32k tokens, 64 heads: 15.0 to 15.5 ms, 1130 to 1170 TFLOP/s; 8k, 32
// heads: 0.50 ms, 1110), many short ones the instructions that find a block and start and end it, single short ones latencies (37 tokens: 5.6 us in a graph).
#include "kvc_prompt_internal.h"
#include "../../include/kvc.h"

#include <math.h>

namespace kvc {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bhalf2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kGroup = 32;                   // tokens of a product with values
constexpr float kSlack = 7.0f;
// A weight's exponent is score * factor + shift, one instruction, with the shift rounded to 32 bits: all weights of a row are off by one power of two, which
// their sum has too, but which has to stay small.  Rows whose maximum is further from zero than this take it from the scores themselves (fp16 rows
// with scores from 2^27 would leave the type, bf16 ones from 2^31).  (What the looking costs: 1 % at 8k tokens, 32 heads, 4 % at 1k.)
constexpr float kFar = 65536.0f;
// Weights are 2^(bias + score - maximum), where the maximum may be up to kSlack below the row's own: fp16 ones as large as the type allows (2^15 with the
// slack), so that those down to 2^-32 of the largest count (2^-39 where all the slack is used), bf16 ones small (2^-20 with the slack), so that sums of
// 2^20 times the largest values stay inside 32 bits (values below 2^-99 lose bits for it).
template <int DT> constexpr float kBias = DT == DT_F16 ? 8.0f : -27.0f;
constexpr float kNone = -__builtin_inff();
template <int DT> constexpr float kLargest = DT == DT_F16 ? 65504.0f : 3.38953139e38f;       // of the type
// Weights of up to this many tokens are added up in 32 bits (a tile's as a tree, then tile by tile: 20 roundings at most), sums of these in 64
// bits.  Added one by one over a long prompt, equal weights round the same way each time: 32k of them were off by 0.00012, 128k by 0.0005.  (8k
// tokens, 32 heads: 495 us, one by one 491.)
constexpr int kFold = 512;
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
template <int N> __device__ __forceinline__ int turned_lane(int x) { return __builtin_amdgcn_update_dpp(0, x, 0x120 + N, 0xf, 0xf, true); }
__device__ __forceinline__ int sum_of_wave(int x)
{
    x += turned_lane<8>(x);
    x += turned_lane<4>(x);
    x += turned_lane<2>(x);
    x += turned_lane<1>(x);
    auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = (int)(a[0] + a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __builtin_amdgcn_readfirstlane((int)(b[0] + b[1]));
}

// ---- which block ------------------------------------------------------------------------------------

struct Block {
    int row0, rows;                          // of the sequence
    int first;                               // of the block, in the sequence
    long long all;                           // blocks of the call
};

// The workgroup that reports.
__device__ __forceinline__ bool first_group() { return blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0; }
// Rows of sequence s, none where its numbers do not fit (reported).
__device__ __forceinline__ int rows_of(const PromptArgs &a, int s, int &row0)
{
    row0 = a.start[s];
    const int rows = (int)((unsigned)a.start[s + 1] - (unsigned)row0);
    if (row0 >= 0 && (unsigned)rows <= (unsigned)a.max_rows && (long long)row0 + rows <= a.rows) return rows;
    if (first_group() && threadIdx.x < 64) atomicOr(a.status + s, KVC_DEV_BAD_ROW);
    return 0;
}

// Block `number` of up to 64 * EACH sequences, longest first (those with most tokens before them, over all sequences).
template <int EACH> __device__ __forceinline__ bool find_sorted(const PromptArgs &a, int number, int size, Block &b)
{
    const int lane = lane_id();
    int blocks[EACH], rows[EACH], row0[EACH], all = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int s = 64 * i + lane;
        rows[i] = row0[i] = 0;
        if (s < a.n) rows[i] = rows_of(a, s, row0[i]);
        blocks[i] = (int)((unsigned)(rows[i] + size - 1) / (unsigned)size);
        all += blocks[i];
    }
    all = sum_of_wave(all);
    b.all = all;
    if (number >= all) return false;
    // the highest level (blocks before it in its sequence) at and above which there are more than `number` blocks
    int low = 0, above = 0;                  // (low: more than `number`; the next that was tried: `above`, which is no more)
    for (int step = 1 << (31 - __builtin_clz(((unsigned)a.max_rows + size - 1) / size | 1u)); step; step >>= 1) {
        const int level = low + step;
        int sum = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) sum += blocks[i] > level ? blocks[i] - level : 0;
        sum = sum_of_wave(sum);
        if (sum > number) low = level;
        else above = sum;
    }
    // Of the last level tried above `low` no more than `number` blocks are there; of the sequences that have one at `low`, in their order:
    int left = number - above;
    b.first = low * size;
    b.row0 = b.rows = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const unsigned long long have = __ballot(blocks[i] > low);
        const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(have >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)have, 0));
        const unsigned long long it = __ballot(blocks[i] > low && before == left);
        if (it) {
            const int l = __ffsll(it) - 1;
            b.row0 = __builtin_amdgcn_readlane(row0[i], l);
            b.rows = __builtin_amdgcn_readlane(rows[i], l);
        }
        left -= __popcll(have);
    }
    return true;
}

// Block `number` of all blocks of `size` rows, the same in all lanes; false where there are fewer.  The blocks of up to kSorted sequences
// come longest first, so that the last ones to run are short; those of more sequences in the order of the sequences, each from its end.
__device__ __forceinline__ bool find_block(const PromptArgs &a, long long number, int size, Block &b)
{
    const int lane = lane_id();
    if (a.n == 1) {
        b.rows = __builtin_amdgcn_readfirstlane(rows_of(a, 0, b.row0));
        b.row0 = __builtin_amdgcn_readfirstlane(b.row0);
        b.all = (unsigned)(b.rows + size - 1) / (unsigned)size;
        b.first = (int)(b.all - 1 - number) * size;
        return number < b.all;
    }
    // (2^30 blocks at most: rows are no more than 2^28, blocks no less than 64)
    if (a.n <= 64) return find_sorted<1>(a, (int)number, size, b);
    if (a.n <= kSorted) return find_sorted<kSorted / 64>(a, (int)number, size, b);
    // kSorted sequences at a time, whose sum says whether the block is among them (300 prompts of 30 tokens, 32 heads: 78 us, 200: 43; 700: 238.  With
    // the starts held in registers 70 and 216, but one prompt of 8k tokens 0.5 % more, for the registers)
    bool found = false;
    b.row0 = b.rows = b.first = 0;
    b.all = 0;
    for (int begin = 0; begin < a.n; begin += kSorted) {
        int sums = 0, row0;
#pragma unroll
        for (int i = 0; i < kSorted; i += 64)
            if (begin + i + lane < a.n) sums += (unsigned)(rows_of(a, begin + i + lane, row0) + size - 1) / (unsigned)size;
        sums = sum_of_wave(sums);
        if (!found && number < b.all + sums) {
            int left = (int)(number - b.all);
            found = true;
#pragma clang loop unroll(disable)
            for (int i = 0; i < kSorted && left >= 0; i += 64) {
                const int s = begin + i + lane;
                int rows = 0;
                row0 = 0;
                if (s < a.n) rows = rows_of(a, s, row0);
                int sum = (int)((unsigned)(rows + size - 1) / (unsigned)size);         // of the sequences up to the lane's
#pragma clang loop unroll(disable)
                for (int d = 1; d < 64; d <<= 1) {
                    const int up = __shfl_up(sum, d, 64);
                    if (lane >= d) sum += up;
                }
                const unsigned long long behind = __ballot(sum > left);
                const int many = __builtin_amdgcn_readlane(sum, 63);
                if (behind) {
                    const int l = __ffsll(behind) - 1;
                    b.row0 = __builtin_amdgcn_readlane(row0, l);
                    b.rows = __builtin_amdgcn_readlane(rows, l);
                    b.first = (__builtin_amdgcn_readlane(sum, l) - 1 - left) * size;
                    left = -1;
                } else left -= many;
            }
        }
        b.all += sums;
    }
    return found;
}

template <bool B> struct BoolConst {
    static constexpr bool value = B;
};

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

// A value that nothing computed from it is moved away from: what a loop needs is made in front of that loop and not held through another.
__device__ __forceinline__ int here_only(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}
#define in_lds __attribute__((address_space(3)))
__device__ __forceinline__ uint32_t lds_address(const u32x4 *x) { return (uint32_t)(uintptr_t)(const in_lds u32x4 *)x; }
// 16 bytes per lane from global memory into the wave's 1 KB of LDS.  (Written out: for the builtin the compiler waits until nothing is on its way
// to LDS before every transposing load.  There is no register that the load would write; wait_for_tiles waits.)
__device__ __forceinline__ void copy_to_lds(const char *from, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(offset), "s"(from) : "memory");
}
// Everything that this wave has requested for LDS is there, and everything that the other waves have.
__device__ __forceinline__ void wait_for_tiles()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// TILES: of 16 rows per wave.  TOKENS: of a tile of K and V in LDS, 64 or 32.  TURNS: sets of kPromptWaves waves, each of which has all rows of
// the block and takes every TURNS-th tile; the second set's results are joined to the first's in the end.
template <int DT, int TILES, int TOKENS, int TURNS>
__global__ __launch_bounds__(64 * kPromptWaves * TURNS, TOKENS == 32 && TILES == 1 ? 4 : TOKENS == 32 ? 3 : 2) void prompt_kernel(PromptArgs a)
{
    constexpr int kRows = 16 * TILES, kBlock = kRows * kPromptWaves, kPieces = TOKENS * 16, kHalves = TOKENS / kGroup;
    constexpr int kLoads = kPieces / (64 * kPromptWaves);         // pieces of a tile that a lane brings
    __shared__ __attribute__((aligned(256))) u32x4 room[TURNS * 4 * kPieces];
    // sums of weights before the last kFold tokens, here because a register each is more than there is (read and written every kFold tokens)
    __shared__ double sums_before[TILES][64 * kPromptWaves * TURNS];
    const int lane = lane_id(), turn = wave_id() / kPromptWaves, wave = wave_id() % kPromptWaves, i = lane & 15, g = lane >> 4;
    u32x4 *keys = room + turn * 4 * kPieces, *values = keys + 2 * kPieces;       // two tiles of each
    // neighbouring workgroups, which run on different XCDs, have different KV heads; those of one KV head meet in an L2
    const int q_heads = a.kv_heads * a.per_kv, kv = blockIdx.x, head = kv * a.per_kv + blockIdx.y;
    for (long long number = blockIdx.z;; number += gridDim.z) {
        Block b;
        if (!find_block(a, number, kBlock, b)) return;
        const int first = b.first + wave * kRows;                  // of the wave
        const uint16_t *q_at = a.q + (long long)b.row0 * a.q_row + head * a.q_head;
        const uint16_t *k_at = a.k + (long long)b.row0 * a.k_row + kv * a.k_head;
        const uint16_t *v_at = a.v + (long long)b.row0 * a.v_row + kv * a.v_head;
        const int tokens = b.first + kBlock < b.rows ? b.first + kBlock : b.rows;
        const int tiles = (tokens + TOKENS - 1) / TOKENS;
        // A tile of keys or values into its half of LDS: the lane's places in LDS are fixed (64 lanes have 1 KB in a row), so the
        // octets are turned by what each lane asks for.  An address is one of the wave and an offset of the lane's that stays.  In place of
        // tokens behind the sequence there is the tile's first, which no row sees.
        const int place_in = wave * 4 + g;             // (of 16 tokens; lane g * 16 + i brings piece i)
        const uint32_t key_at = place_in * 2 * (uint32_t)a.k_row + 16 * (key_piece(place_in, i) & 15);
        const uint32_t value_at = place_in * 2 * (uint32_t)a.v_row + 16 * (value_piece(place_in, i) & 15);
        struct Stream {
            const char *at;                  // of its next tile
            int n;
        };
        auto bring = [&](Stream &next, u32x4 *tile, long long stride, uint32_t lane_at) {
            if (next.n >= tiles) return;
            const int have = b.rows - next.n * TOKENS;
            const uint32_t to = lds_address(tile + (next.n / TURNS & 1) * kPieces + wave * 64);
            if (have >= TOKENS) {
                const char *at = next.at;
#pragma unroll
                for (int r = 0; r < kLoads; ++r, at += 32 * stride) copy_to_lds(at, lane_at, to + r * kPromptWaves * 1024);
            } else {
                const uint32_t own = here_only(place_in), step = 32 * (uint32_t)stride;
#pragma unroll
                for (int r = 0; r < kLoads; ++r) {
                    const bool there = (int)own < have - r * 16;
                    copy_to_lds(next.at, there ? lane_at + r * step : lane_at - own * 2 * (uint32_t)stride, to + r * kPromptWaves * 1024);
                }
            }
            next.at += TURNS * TOKENS * 2 * stride;
            next.n += TURNS;
        };
        Stream next_key, next_value;
        auto bring_key = [&]() { bring(next_key, keys, a.k_row, key_at); };
        auto bring_value = [&]() { bring(next_value, values, a.v_row, value_at); };
        auto bring_first = [&]() {
            next_key = {(const char *)(k_at + (long long)turn * TOKENS * a.k_row), turn};
            next_value = {(const char *)(v_at + (long long)turn * TOKENS * a.v_row), turn};
            bring_key();
            bring_value();
            bring_key();
        };
        bring_first();
        // (behind the first tiles, whose requests the compiler does not count: it waits for these, which come last)
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
        float top[TILES], shift[TILES], sum[TILES], size[TILES];       // top: of the scores without the factor; size: sum of the lane's results' magnitudes
        bool far = false;                                     // some row of the wave is (kFar)
        auto is_far = [&](float x) { return fabsf(x * a.factor) > kFar; };
        // Tile n.  MIXED: some rows see some of its tokens only, or none.  AGAIN: with values that are not finite taken out where they are
        // not seen.
        auto do_tile = [&](int n, int lane, auto mixed_tile, auto second_time) {
            const int i = lane & 15, g = lane >> 4;
            constexpr bool MIXED = decltype(mixed_tile)::value, AGAIN = decltype(second_time)::value;
            // (turning an octet by a token's number is an exclusive or, and the tiles lie at multiples of their rows: all octets' addresses
            // are the first one's and an exclusive or with a constant)
            const uint32_t key_lane = lds_address(keys + (n / TURNS & 1) * kPieces) + 16 * key_piece(i, g);
            const uint32_t value_lane = lds_address(values + (n / TURNS & 1) * kPieces) + 16 * value_piece(4 * g + (i >> 2), (i & 3) >> 1) + 8 * (i & 1);
            const int token = n * TOKENS;
            const bool some = !MIXED || (first < b.rows && token < first + kRows && (TURNS == 1 || n < tiles)), both = !MIXED || token + kGroup < first + kRows;
            u32x4 weight[kHalves][TILES];
            if (some) {
                f32x4 score[2 * kHalves][TILES];
#pragma unroll
                for (int h = 0; h < 2 * kHalves; ++h) {
#pragma unroll
                    for (int t = 0; t < TILES; ++t) score[h][t] = f32x4{0, 0, 0, 0};
                    if (h >= 2 && !both) continue;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const u32x4 key = *(const in_lds u32x4 *)(uintptr_t)((key_lane ^ 64 * c) + 4096 * h);       // token 16 h + i, octet 4 c + g
#pragma unroll
                        for (int t = 0; t < TILES; ++t) score[h][t] = multiply<DT>(key, query[t][c], score[h][t]);
                    }
                }
                if (MIXED) {
#pragma unroll
                    for (int h = 0; h < 2 * kHalves; ++h)
#pragma unroll
                        for (int t = 0; t < TILES; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (token + 16 * h + 4 * g + e > first + 16 * t + i) score[h][t][e] = kNone;
                }
                bool grown = false;
                float most[TILES];
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    most[t] = score[0][t][0];
#pragma unroll
                    for (int e = 1; e < 8 * kHalves; ++e) most[t] = fmaxf(most[t], score[e >> 2][t][e & 3]);
                    grown |= (most[t] - top[t]) * a.factor > kSlack;
                }
                if (__any(grown)) {
                    bool some_far = false;
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        // (rows that have not grown stay as they are: a row's bits depend on what it sees alone)
                        const float highest = max_of_row(most[t]);
                        const float now = (highest - top[t]) * a.factor > kSlack ? highest : top[t];
                        const float from = now == kNone ? 0.0f : now;
                        const float by = __builtin_amdgcn_exp2f((top[t] - from) * a.factor);
                        top[t] = now;
                        shift[t] = is_far(from) ? kBias<DT> : __builtin_fmaf(-from, a.factor, kBias<DT>);
                        some_far |= is_far(from);
                        sum[t] *= by;
                        if (n >= kFold / TOKENS * TURNS) sums_before[t][threadIdx.x] *= by;
#pragma unroll
                        for (int d = 0; d < 8; ++d) out[t][d] *= by;
                    }
                    far = __any(some_far);
                }
                if (__builtin_expect(far, false)) {
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        const float off = top[t] != kNone && is_far(top[t]) ? top[t] : 0.0f;
#pragma unroll
                        for (int h = 0; h < 2 * kHalves; ++h) score[h][t] -= off;
                    }
                }
                float part[kHalves][TILES];
#pragma unroll
                for (int h = 0; h < 2 * kHalves; ++h)
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        float w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(score[h][t][e], a.factor, shift[t]));
                        const float four = (w[0] + w[1]) + (w[2] + w[3]);
                        part[h >> 1][t] = h & 1 ? part[h >> 1][t] + four : four;
                        weight[h >> 1][t][2 * (h & 1)] = round_pair<DT>(w[0], w[1]);
                        weight[h >> 1][t][2 * (h & 1) + 1] = round_pair<DT>(w[2], w[3]);
                    }
#pragma unroll
                for (int t = 0; t < TILES; ++t) sum[t] += kHalves > 1 ? part[0][t] + part[kHalves - 1][t] : part[0][t];
                if ((n / TURNS + 1) % (kFold / TOKENS) == 0) {
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        sums_before[t][threadIdx.x] += sum[t];
                        sum[t] = 0.0f;
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < TILES; ++t) asm volatile("" : "+v"(sum[t]));   // (added up here, not held apart until the products are done)
            wait_for_tiles();                        // this tile's values, the next tile's keys
            // (what the next ones overwrite has no readers behind the barrier: this tile's keys, the last tile's values)
            bring_value();
            bring_key();
            // token 4 g + i / 4 of the lane's 16 (then 16 further), channels 16 d + 4 (i % 4) ... + 3; the lane gets tokens
            // 4 g ... 4 g + 3 of channel 16 d + i
            auto value_of = [&](int half, int d) {
                u32x4 value;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (in_lds s16x4 *)(uintptr_t)((value_lane ^ 32 * d) + 8192 * half + 4096 * h)));
                    value[2 * h] = x[0];
                    value[2 * h + 1] = x[1];
                }
                return value;
            };
            if (some) {
#pragma unroll
                for (int half = 0; half < kHalves; ++half) {
                    if (half && !both) continue;
                    u32x4 seen[TILES];
                    if (MIXED && AGAIN) {
                        constexpr uint32_t one = DT == DT_F16 ? 0x3c00u : 0x3f80u;
#pragma unroll
                        for (int t = 0; t < TILES; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int behind = first + 16 * t + i - (token + 32 * half + 16 * (e >> 1) + 4 * g + 2 * (e & 1));
                                seen[t][e] = (behind >= 0 ? one : 0u) | (behind >= 1 ? one << 16 : 0u);
                            }
                    }
#pragma unroll
                    for (int d = 0; d < 8; ++d) {
                        u32x4 value = value_of(half, d), lost;
                        if (MIXED && AGAIN) only_finite<DT>(value, lost);
#pragma unroll
                        for (int t = 0; t < TILES; ++t) {
                            if (MIXED && AGAIN) {
                                const f32x4 count = multiply<DT>(lost, seen[t], f32x4{0, 0, 0, 0});
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (count[e] > 0.0f) out[t][d][e] = __builtin_nanf("");
                            }
                            out[t][d] = multiply<DT>(value, weight[half][t], out[t][d]);
                        }
                    }
                }
            }
        };
        auto do_tiles = [&](auto second_time) {
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                top[t] = kNone;
                shift[t] = kBias<DT>;
                sum[t] = 0.0f;
                far = false;
                sums_before[t][threadIdx.x] = 0.0;
#pragma unroll
                for (int d = 0; d < 8; ++d) out[t][d] = f32x4{0, 0, 0, 0};
            }
            if (decltype(second_time)::value) bring_first();
            wait_for_tiles();
            // (all sets pass the same barriers: a set may have a tile behind the last one, of which no row sees anything)
            const int whole = b.first / TOKENS / TURNS * TURNS;       // tiles of which all rows see all tokens
            const int for_whole = here_only(lane);
            for (int n = 0; n < whole; n += TURNS) do_tile(n + turn, for_whole, BoolConst<false>(), second_time);
            const int for_mixed = here_only(lane);
            for (int n = whole; n < tiles; n += TURNS) do_tile(n + turn, for_mixed, BoolConst<true>(), second_time);
            if (tiles > (kFold / TOKENS - 1) * TURNS) {
#pragma unroll
                for (int t = 0; t < TILES; ++t) sum[t] = (float)(sums_before[t][threadIdx.x] + sum[t]);
            }
            if constexpr (TURNS > 1) {
                constexpr int kResults = TILES * 8 * kPromptWaves * 64, kStatistics = TILES * kPromptWaves * 64;       // of a set
                static_assert((TURNS - 1) * (kResults * sizeof(f32x4) + kStatistics * sizeof(f32x2)) <= sizeof(room), "results go through the tiles' room");
                f32x4 *results = (f32x4 *)room + wave * 64 + lane;
                f32x2 *statistics = (f32x2 *)((f32x4 *)room + (TURNS - 1) * kResults) + wave * 64 + lane;
                __syncthreads();
                if (turn) {
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        statistics[(turn - 1) * kStatistics + t * kPromptWaves * 64] = f32x2{top[t], sum[t]};
#pragma unroll
                        for (int d = 0; d < 8; ++d) results[(turn - 1) * kResults + (t * 8 + d) * kPromptWaves * 64] = out[t][d];
                    }
                }
                __syncthreads();
                if (turn) return true;
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int k = 0; k < TURNS - 1; ++k) {
                        const f32x2 other = statistics[k * kStatistics + t * kPromptWaves * 64];
                        const float now = fmaxf(top[t], other[0]), from = now == kNone ? 0.0f : now;
                        const float by = __builtin_amdgcn_exp2f((top[t] - from) * a.factor), other_by = __builtin_amdgcn_exp2f((other[0] - from) * a.factor);
                        top[t] = now;
                        shift[t] = is_far(from) ? kBias<DT> : __builtin_fmaf(-from, a.factor, kBias<DT>);
                        sum[t] = sum[t] * by + other[1] * other_by;
#pragma unroll
                        for (int d = 0; d < 8; ++d) out[t][d] = out[t][d] * by + results[k * kResults + (t * 8 + d) * kPromptWaves * 64] * other_by;
                    }
            }
            bool finite = true;
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                f32x4 sums = {0, 0, 0, 0};
#pragma unroll
                for (int d = 0; d < 8; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sums[e] += fabsf(out[t][d][e]);
                size[t] = sums[0] + sums[1] + (sums[2] + sums[3]);
                finite &= size[t] < -kNone;
            }
            return finite || first >= b.rows;
        };
        const bool finite = do_tiles(BoolConst<false>());
        if (__builtin_amdgcn_readfirstlane(__syncthreads_or(!finite))) do_tiles(BoolConst<true>());
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            if (turn) break;
            const int row = first + 16 * t + i;
            const float all = sum_of_row(sum[t]), by = 1.0f / all;
            if (row >= b.rows) continue;
#pragma unroll
            for (int d = 0; d < 8; ++d) out[t][d] *= by;
            // A mean of numbers of the type that is beyond them is there by its weights' roundings.  (Looked at where the lane's sum of magnitudes is.)
            if (__builtin_expect(__any(!(size[t] * by <= kLargest<DT>)), false)) {
#pragma unroll
                for (int d = 0; d < 8; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (fabsf(out[t][d][e]) < -kNone) out[t][d][e] = fminf(fmaxf(out[t][d][e], -kLargest<DT>), kLargest<DT>);
            }
            uint16_t *to = a.out + (long long)(b.row0 + row) * a.o_row + head * a.o_head + 4 * here_only(g);
#pragma unroll
            for (int d = 0; d < 8; ++d) *(u32x2 *)(to + 16 * d) = u32x2{round_pair<DT>(out[t][d][0], out[t][d][1]), round_pair<DT>(out[t][d][2], out[t][d][3])};
            if (a.lse && g == 0)
                a.lse[(long long)(b.row0 + row) * q_heads + head] = (__builtin_amdgcn_logf(all) - shift[t] + (is_far(top[t]) ? top[t] * a.factor : 0.0f)) * 0.693147181f;
        }
        if (number + gridDim.z >= b.all) return;
        __syncthreads();
    }
}

// ---- which kernel ---------------------------------------------------------------------------------

// The kernels, and what a call takes with each, us: the longest sequence's tiles one after the other (per 64 tokens), the products at the rate of a
// full chip, what a workgroup takes apart from them, and the launch.  Times of calls in the sizes, us, tokens x heads:
//   64 rows    37 x 64 5.8, 64 x 100 x 32 38, 1024 x 64 33                                          tiles of 32 tokens, four workgroups per compute unit
//   64 shared  512 x 32 13.5 (one set of waves 17.0), 1024 x 32 22.3 (29.3), 4096 x 8 64 (98)   two sets of waves take turns: too few rows for the chip
//   128 rows   2048 x 64 83 (64 rows: 97), 4096 x 32 155 (175), 8 x 1024 x 32 99 (106)             tiles of 32 tokens, three workgroups
//   192 rows   8192 x 32 503 (128 rows: 517), 32768 x 64 15.1 ms (16.2)                              tiles of 64 tokens, two workgroups: K and V are read least
// The numbers are fitted to the choice among 150 measured calls (1 to 128 sequences of 16 to 32k tokens, 8 to 64 heads, bf16): its
// time is 0.6 % above the least in the mean, 13 % at worst; of 110 others (fp16) 0.7 and 15 % (profiles/prompt_block_rows.txt).
struct Kernel {
    int tiles, tokens, turns;
    float per_64, rate, group, launch;       // us, TFLOP/s, us, us
};
constexpr Kernel kKernels[] = {{1, 32, 1, 1.29f, 920.0f, 0.0069f, 5.0f},
                               {1, 32, 2, 0.82f, 810.0f, 0.0116f, 5.6f},
                               {2, 32, 1, 1.80f, 1150.0f, 0.0137f, 5.2f},
                               {3, 64, 1, 1.80f, 1185.0f, 0.0244f, 6.5f}};
constexpr int kKinds = sizeof(kKernels) / sizeof(kKernels[0]);

// Blocks of `size` rows that a call has at most: what the sequences' number and bound allow, or their rows in all.
static long long most_blocks(const PromptArgs &a, int size)
{
    const long long each = ((long long)a.max_rows + size - 1) / size * a.n, rows = a.rows / size + a.n;
    return each < rows ? each : rows;
}
static int kernel_for(const PromptArgs &a)
{
    const double heads = (double)a.kv_heads * a.per_kv, longest = a.max_rows < a.rows ? a.max_rows : (double)a.rows;
    const double rows = (double)a.max_rows * a.n < a.rows ? (double)a.max_rows * a.n : (double)a.rows;
    // (of equal sequences; of ragged ones an estimate between those of the longest and of the mean)
    const double pairs = rows * (longest + rows / a.n) / 4;
    int best = 0;
    double least = 0.0;
    for (int k = 0; k < kKinds; ++k) {
        const Kernel &c = kKernels[k];
        const double chain = c.per_64 * longest / 64, groups = heads * most_blocks(a, 16 * c.tiles * kPromptWaves);
        const double work = 4.0 * kDim * heads * pairs / c.rate * 1e-6 + c.group * groups;
        const double time = c.launch + sqrt(chain * chain + work * work);
        if (k == 0 || time < least) {
            best = k;
            least = time;
        }
    }
    return best;
}

template <int DT, int KIND> static void launch_kind(const PromptArgs &a, hipStream_t stream)
{
    constexpr Kernel c = kKernels[KIND];
    // (a grid has 65535 places in this direction; further blocks are taken in turn, which also covers starts that overlap)
    const long long blocks = most_blocks(a, 16 * c.tiles * kPromptWaves);
    const dim3 grid(a.kv_heads, a.per_kv, (unsigned)(blocks < 1 ? 1 : blocks > 65535 ? 65535 : blocks));
    prompt_kernel<DT, c.tiles, c.tokens, c.turns><<<grid, 64 * kPromptWaves * c.turns, 0, stream>>>(a);
}
template <int DT> static void launch_type(const PromptArgs &a, int kind, hipStream_t stream)
{
    if (kind == 0) launch_kind<DT, 0>(a, stream);
    else if (kind == 1) launch_kind<DT, 1>(a, stream);
    else if (kind == 2) launch_kind<DT, 2>(a, stream);
    else launch_kind<DT, 3>(a, stream);
}
void launch_prompt(int dtype, const PromptArgs &a, hipStream_t stream)
{
    if (dtype == DT_F16) launch_type<DT_F16>(a, kernel_for(a), stream);
    else launch_type<DT_BF16>(a, kernel_for(a), stream);
}

int prompt_block_rows(const PromptArgs &a, int &waves)
{
    const Kernel &c = kKernels[kernel_for(a)];
    waves = kPromptWaves * c.turns;
    return 16 * c.tiles * kPromptWaves;
}

}  // namespace kvc
