// Host-side declarations shared by the translation units of the quantised cache.
#pragma once

#include "kvc_cache.h"

namespace kvc {

template <int N> struct IntConst {
    static constexpr int value = N;
};

struct CacheTypes {
    int dtype, bits_k, bits_v, group;
    bool rotate;                   // K rows and queries
};

// Workgroups of 256 threads per sequence of a call that stores or loads rows.
long long row_places(const CacheView &c);
void launch_cache_rows(const CacheTypes &t, const CacheView &c, bool store, uint16_t *k, uint16_t *v, long long stride_row,
                       long long stride_head, int n, hipStream_t stream);
void launch_cache_keep(const CacheTypes &t, const CacheView &c, const int *keep_start, const int *keep, int max_keep, int n,
                       hipStream_t stream);

// Arguments of the attention kernels.
struct AttendArgs {
    CacheView c;
    const uint16_t *q;
    uint16_t *out;
    float *lse;                    // or null
    // sequences in several parts: sums of a part's rows, [slot][128], (maximum, sum of weights), [slot][2], and how many of
    // a sequence's parts are done (zero between the calls)
    float *part, *part_ml;
    int *counters;
    long long part_rows;           // rows that the results have room for (below 2^32 bytes)
    long long q_row, q_head, o_row, o_head;        // strides in elements
    float scale;                   // of the scores
    // the division of sequences (see find_part), in the tokens that a workgroup's waves take at a time: whether there is one, workgroups
    // per head and block of rows that the chip holds at once, what cutting has to gain, what joining takes per piece, and how much
    // longer a workgroup takes beside another one (0: there is none)
    int divide, parts, joining;
    float joining_piece, alone;
    int per_kv;                    // query heads per KV head
    int row_blocks;                // of 16 * tiles query rows, in the longest sequence
    int n;
    int dtype, rotate;
};

constexpr int kMostDivided = 256;             // sequences of a call whose sequences are divided
constexpr int kWideRows = 128, kWideTiles = kWideRows / 16;

// The attention of one pair of code widths (10 * bits_k + bits_v) with 1 or 2 tiles of 16 query rows per workgroup, or (kWideTiles) 128
// rows; `places` workgroups.
template <int BITS> void launch_attend(const CacheTypes &t, const AttendArgs &a, int tiles, int places, hipStream_t stream);
template <> void launch_attend<44>(const CacheTypes &, const AttendArgs &, int, int, hipStream_t);
template <> void launch_attend<48>(const CacheTypes &, const AttendArgs &, int, int, hipStream_t);
template <> void launch_attend<84>(const CacheTypes &, const AttendArgs &, int, int, hipStream_t);
template <> void launch_attend<88>(const CacheTypes &, const AttendArgs &, int, int, hipStream_t);

}  // namespace kvc
