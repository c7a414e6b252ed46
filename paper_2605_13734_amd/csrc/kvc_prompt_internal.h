// Host-side declarations shared by the translation units of the calls on prompts (rotation, attention) and on the pages' tables.
#pragma once

#include "kvc_device.h"

namespace kvc {

// ---- queries and keys, normed and rotated ---------------------------------------------------------

constexpr int kMostPairs = kDim / 2;

// Two 16-bit tensors of rows of heads: read from one place, written to another (or the same).
struct RotateTensor {
    const uint16_t *in, *weight;   // weight: null where heads are not normed
    uint16_t *out;
    long long in_row, in_head, out_row, out_head;      // strides in elements
    int heads;                     // 0: the tensor is not there
    int pad;
};

// Arguments of the rotation (members of whole words only).
struct RotateArgs {
    RotateTensor q, k;
    const int *positions;
    long long rows;
    uint64_t turns[kMostPairs];    // of a pair per position, in 2^-64 of a turn
    float eps, amplitude;
    int pairs;                     // rotated pairs of channels, a multiple of 8
    int chunk, chunks;             // heads of a row that a wave takes, waves per row
    int past_caches, pad;          // rows are read past the caches
};

// Divides the rows (chunk, chunks, past_caches of the arguments): a wave has one row and one chunk, a workgroup four waves.
void divide_rows(RotateArgs &a);
void launch_rotate(int dtype, bool neighbours, bool norm, const RotateArgs &a, long long groups, hipStream_t stream);

// ---- attention over whole prompts ------------------------------------------------------------------

struct PromptArgs {
    const uint16_t *q, *k, *v;
    uint16_t *out;
    float *lse;                    // or null
    const int *start;
    int *status;
    long long rows;
    long long q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;       // strides in elements
    float factor;                  // of the scores, times log2(e): above zero
    uint32_t query_and, query_xor; // what is done to pairs of queries: signs turned for a scale below zero, cleared for zero
    int n, max_rows, kv_heads, per_kv;
};

constexpr int kPromptWaves = 4;               // that divide the rows of a block

void launch_prompt(int dtype, const PromptArgs &a, hipStream_t stream);
// rows of a block, and waves of a workgroup, in a call with these bounds
int prompt_block_rows(const PromptArgs &a, int &waves);

// ---- the pages' tables -----------------------------------------------------------------------------

struct AdvanceArgs {
    int *held, *block_table, *free_pages, *new_start, *tokens, *positions, *status;
    const int *kept, *fresh;
    long long *slots;
    long long table_stride, rows;
    int n, max_new, max_tokens, num_pages, page_shift;
};

void launch_advance(const AdvanceArgs &a, hipStream_t stream);

}  // namespace kvc
