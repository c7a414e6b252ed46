// Host side of the quantised cache: plans, checks of the arguments, how the attention's work is divided.
#include "kvc_cache_internal.h"
#include "../../include/kvc.h"

#include <new>

struct kvc_cache_plan_s {
    kvc_cache_config config;
    int64_t max_tokens;
    int32_t max_new, max_batch;
    size_t page_bytes, workspace;
};

namespace kvc {

// Workgroups that the chip holds, as the kernels' registers have it: one of 8 or 12 waves per compute unit for blocks of 16 and 32 rows,
// two of 4 waves for blocks of 128 (8 trees of 64 drafts over 8k tokens, 8 x 8 heads, divided among 512 / 768 / 1024: 293 / 344 / 321 us).
constexpr int kFewGroups = 256, kManyGroups = 512;
// What cutting sequences has to gain, in steps of a workgroup's waves, and what joining takes per piece (128 rows: 64 KB, read by one
// workgroup; with few rows per 16 of them).  One sequence, one token, steps that cutting has to gain 1 / 2 / 3: 1k tokens 11.0 / 11.0 / 11.3 us;
// 8 drafts over 4k in blocks of 32, per piece and 16 rows 0.025 / 0.05: 18.4 / 16.5 us, one token over 16k 0.02 / 0.05 / 0.1: 16.7 / 16.7 / 17.6; 64
// drafts in blocks of 128, per piece 0.1 / 0.3 / 0.5 / 1: over 4k 44.3 / 39.3 / 42.4 / 45.7, over 64k - / 161 / 162 / 189 us.
constexpr int kFewJoining = 2, kManyJoining = 4;
constexpr float kFewJoiningPiece = 0.05f, kManyJoiningPiece = 0.3f;
constexpr float kManyAlone = 1.5f;           // 64 drafts over 16k tokens in blocks of 128: 18 pieces of 7 steps, 288 workgroups, 85 us, 16 of 8 steps 71
constexpr int kLeastDivided = 256;           // tokens: calls of shorter sequences are not divided
constexpr int kCounters = 2 * kManyGroups;   // at the start of the workspace
constexpr size_t kPartBytes = (kDim + 2) * sizeof(float);
constexpr int64_t kMostThreads = 0xffffffffll;       // of a launch, per dimension
constexpr int kMostAttending = 768;                  // threads of an attention's workgroup at most

// How a call's query rows are divided: tiles of 16 rows per workgroup, and what that makes of the tokens.
struct AttendShape {
    int tiles, row_blocks;
    bool divide;
    int64_t parts, places, slots;            // parts per head and block of rows, workgroups, workgroups with results to be joined
};
// The largest tiles that a call with so many rows per sequence and KV head takes.
static int most_tiles(int64_t rows) { return rows <= 16 ? 1 : rows <= 64 ? 2 : kWideTiles; }

// Small blocks of rows read a cache more often and share less of the codes' unpacking, large ones leave more of the chip without work and
// have more to join.  What a call takes was measured for 1 to 16 sequences of 500 to 32k tokens, 8 KV heads, 32 to 512 rows (fp16, 4 bits,
// groups of 32): a time for every 256 (128 rows: 512) blocks at once, and one per block and token (128 rows: per 32 of them, since waves
// without rows leave room).  Blocks of 16 / 32 / 128 rows, us:
// 1 x 64 rows x 2k 13.0 / 15.7 / 26.0; 1 x 128 x 2k 14.2 / 16.1 / 31.4, x 16k 34.1 / 30.5 / 74.1; 1 x 512 x 2k 19.0 / 21.7 / 33.0; 4 x 256 x
// 1k 25.7 / 18.8 / 28.6, x 8k 96.9 / 71.6 / 79.6, x 16k 178 / 134 / 130; 8 x 512 x 500 66.1 / 47.5 / 33.2, x 4k 209 / 154 / 128.
// Of 199 such calls the formulas' choice is the best or within 14 % of it, 0.6 % in the mean; of 90 others, of all widths, types, rotated
// or not, equal and ragged lengths, within 42 %, 2.7 % in the mean (nothing here knows a width, a type or a rotation: rotated 8-bit keys in groups
// of 32 like blocks of 16 better than this does).  Up to 64 rows, blocks of 128 never were the best.  `tokens` is the call's bound, for
// the lengths are on the device: with a bound of 128k the 199 calls take 1.29 times their least in the mean, 3.1 times at worst.
static int tiles_of(int64_t rows, int64_t heads, int64_t tokens)
{
    const int most = most_tiles(rows);
    auto blocks = [&](int size) { return (double)heads * (double)((rows + size - 1) / size); };
    auto times = [](double blocks, double at_once) { return blocks > at_once ? blocks / at_once : 1.0; };
    const double one = blocks(16), two = blocks(32), wide = blocks(kWideRows);
    const double cost_one = 4.5 + 5.0 * times(one, kFewGroups) + 1.9e-5 * one * (double)tokens;
    const double cost_two = 5.0 + 7.0 * times(two, kFewGroups) + 2.9e-5 * two * (double)tokens;
    const double cost_wide = 20.0 + 6.0 * times(wide, kManyGroups) + 2.4e-5 * two * (double)tokens;
    if (most == 1 || (cost_one < cost_two && (most == 2 || cost_one < cost_wide))) return 1;
    return most == 2 || cost_two <= cost_wide ? 2 : kWideTiles;
}

static AttendShape attend_shape(const kvc_cache_config &f, int n, int max_new, int64_t max_tokens)
{
    AttendShape s;
    const int64_t rows = (int64_t)max_new * (f.q_heads / f.kv_heads);
    s.tiles = tiles_of(rows, (int64_t)n * f.kv_heads, max_tokens);
    s.row_blocks = (int)((rows + 16 * s.tiles - 1) / (16 * s.tiles));
    const int64_t each = (int64_t)f.kv_heads * s.row_blocks;
    s.parts = (s.tiles != kWideTiles ? kFewGroups : kManyGroups) / each;
    s.divide = n <= kMostDivided && s.parts > 1 && max_tokens > kLeastDivided;
    // what find_part makes: no more than the parts, or than half of them beyond one piece per sequence; the pieces of sequences that
    // are cut are no more than the parts
    const int64_t other = n + (s.parts + 1) / 2;
    s.places = each * (!s.divide ? n : s.parts > other ? s.parts : other);
    s.slots = s.divide ? each * (s.parts + 1) : 0;
    return s;
}

static CacheTypes types_of(const kvc_cache_config &f)
{
    return CacheTypes{f.dtype, f.bits_k, f.bits_v, f.group, f.transform == KVC_T_HADAMARD};
}

static bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// The checks that all calls share; fills the view.  most_new: the call's bound of new rows.
static int check_call(const kvc_cache_plan_t *plan, const kvc_cache_batch *b, void *pages, int32_t *status, int64_t rows, int64_t most_new,
                      CacheView *c)
{
    if (!plan || !b) return KVC_ERR_ARG;
    const kvc_cache_config &f = plan->config;
    if (b->n < 0 || b->max_new < 0 || b->max_tokens < 0 || b->num_pages < 0 || b->table_stride < 0 || rows < 0) return KVC_ERR_ARG;
    if (b->n > plan->max_batch || b->max_new > most_new || b->max_tokens > plan->max_tokens) return KVC_ERR_CAPACITY;
    if (b->n == 0 || b->max_new == 0 || b->max_tokens == 0) return KVC_OK;
    if (!b->new_start || !b->tokens || !b->block_table || !pages || !status) return KVC_ERR_ARG;
    if (!aligned(b->new_start, 4) || !aligned(b->tokens, 4) || !aligned(b->block_table, 4) || !aligned(status, 4) || !aligned(pages, 16) ||
        !aligned(b->mask, 8)) return KVC_ERR_ARG;
    if (b->table_stride < (b->max_tokens + f.block_tokens - 1) / f.block_tokens) return KVC_ERR_ARG;
    if (b->mask && (int64_t)b->mask_words * 64 < b->max_new) return KVC_ERR_ARG;
    c->pages = (uint8_t *)pages;
    c->new_start = b->new_start;
    c->tokens = b->tokens;
    c->block_table = b->block_table;
    c->mask = (const unsigned long long *)b->mask;
    c->status = status;
    c->table_stride = b->table_stride;
    c->page_bytes = (long long)plan->page_bytes;
    c->rows = rows;
    c->mask_words = b->mask_words;
    c->heads = f.kv_heads;
    c->page_shift = __builtin_ctz((unsigned)f.block_tokens);
    c->num_pages = b->num_pages;
    c->max_new = b->max_new < b->max_tokens ? b->max_new : (int)b->max_tokens;       // (new rows are tokens)
    c->max_tokens = (int)b->max_tokens;
    return KVC_OK;
}

static bool nothing(const kvc_cache_batch *b) { return b->n == 0 || b->max_new == 0 || b->max_tokens == 0; }

static bool strides_ok(int64_t row, int64_t head) { return row % 8 == 0 && head % 8 == 0; }

static int rows_call(const kvc_cache_plan_t *plan, const kvc_cache_batch *batch, const kvc_cache_rows *r, void *pages, int32_t *status,
                     void *stream, bool store)
{
    CacheView c;
    if (!r) return KVC_ERR_ARG;
    const int rc = check_call(plan, batch, pages, status, r->rows, INT32_MAX, &c);
    if (rc != KVC_OK || nothing(batch)) return rc;
    if ((r->rows && (!r->k || !r->v)) || !aligned(r->k, 16) || !aligned(r->v, 16) || !strides_ok(r->stride_row, r->stride_head)) return KVC_ERR_ARG;
    if (row_places(c) > kMostThreads / 256) return KVC_ERR_CAPACITY;
    launch_cache_rows(types_of(plan->config), c, store, (uint16_t *)r->k, (uint16_t *)r->v, r->stride_row, r->stride_head, batch->n,
                      (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? KVC_OK : KVC_ERR_DEVICE;
}

}  // namespace kvc

extern "C" int kvc_cache_plan(const kvc_cache_config *config, int64_t max_tokens, int32_t max_new, int32_t max_batch,
                              kvc_cache_plan_t **out)
{
    using namespace kvc;
    if (!out) return KVC_ERR_ARG;
    *out = nullptr;
    if (!config || max_tokens < 0 || max_new < 1 || max_batch < 1) return KVC_ERR_ARG;
    const kvc_cache_config &f = *config;
    if (f.dtype != KVC_F16 && f.dtype != KVC_BF16) return KVC_ERR_ARG;
    if (f.group != 32 && f.group != 64 && f.group != 128) return KVC_ERR_ARG;
    if (f.kv_heads < 1 || f.q_heads < 1 || f.q_heads % f.kv_heads || f.head_dim < 1 || f.block_tokens < 1) return KVC_ERR_ARG;
    const bool widths = (f.bits_k == 4 || f.bits_k == 8) && (f.bits_v == 4 || f.bits_v == 8);
    const bool pages = f.block_tokens >= kGranule && f.block_tokens <= 4096 && (f.block_tokens & (f.block_tokens - 1)) == 0;
    if (!widths || !pages || f.head_dim != kDim || f.transform > KVC_T_HADAMARD || f.q_heads > 65536 || max_batch > 65535)
        return KVC_ERR_UNSUPPORTED;
    // (row and token numbers are ints in the kernels, and so are the places of a launch)
    if (max_tokens > 0x7fffff00ll || (int64_t)max_new * f.q_heads > 0x3fffffffll) return KVC_ERR_CAPACITY;
    kvc_cache_plan_t *p = new (std::nothrow) kvc_cache_plan_t;
    if (!p) return KVC_ERR_CAPACITY;
    p->config = f;
    p->max_tokens = max_tokens;
    p->max_new = max_new;
    p->max_batch = max_batch;
    p->page_bytes = (size_t)f.kv_heads * (f.block_tokens / kGranule) * granule_map(f.bits_k, f.bits_v, f.group).bytes;
    // the counters, and as many results as a call of up to max_new rows can have (attend_shape: each * (parts + 1) with each * parts of
    // the groups at most and two parts or more, of the largest blocks that such a call may take)
    const int tiles = most_tiles((int64_t)max_new * (f.q_heads / f.kv_heads));
    const size_t slots = (size_t)(tiles == kWideTiles ? kManyGroups : kFewGroups) * 3 / 2;
    p->workspace = max_tokens > kLeastDivided ? slots * 16 * tiles * kPartBytes + kCounters * sizeof(int) : 0;
    *out = p;
    return KVC_OK;
}

extern "C" void kvc_cache_plan_free(kvc_cache_plan_t *plan) { delete plan; }

extern "C" size_t kvc_cache_page_bytes(const kvc_cache_plan_t *plan) { return plan ? plan->page_bytes : 0; }

extern "C" size_t kvc_cache_workspace_size(const kvc_cache_plan_t *plan) { return plan ? plan->workspace : 0; }

extern "C" int32_t kvc_cache_block_rows(const kvc_cache_plan_t *plan, int32_t n, int32_t max_new, int64_t max_tokens)
{
    using namespace kvc;
    if (!plan || n < 1 || max_new < 1 || max_tokens < 1 || n > plan->max_batch || max_new > plan->max_new || max_tokens > plan->max_tokens) return 0;
    return 16 * attend_shape(plan->config, n, max_new < max_tokens ? max_new : (int)max_tokens, max_tokens).tiles;
}

extern "C" int kvc_cache_store(const kvc_cache_plan_t *plan, const kvc_cache_batch *batch, const kvc_cache_rows *rows, void *pages,
                               int32_t *dev_status, void *hip_stream)
{
    return kvc::rows_call(plan, batch, rows, pages, dev_status, hip_stream, true);
}

extern "C" int kvc_cache_load(const kvc_cache_plan_t *plan, const kvc_cache_batch *batch, const kvc_cache_rows *rows, const void *pages,
                              int32_t *dev_status, void *hip_stream)
{
    return kvc::rows_call(plan, batch, rows, (void *)pages, dev_status, hip_stream, false);
}

extern "C" int kvc_cache_keep(const kvc_cache_plan_t *plan, const kvc_cache_batch *batch, const int32_t *keep_start, const int32_t *keep,
                              int64_t keep_rows, void *pages, int32_t *dev_status, void *hip_stream)
{
    using namespace kvc;
    CacheView c;
    const int rc = check_call(plan, batch, pages, dev_status, INT64_MAX, INT32_MAX, &c);
    if (rc != KVC_OK || nothing(batch)) return rc;
    if (!keep_start || (keep_rows && !keep) || keep_rows < 0 || keep_rows > 0x7fffffffll || !aligned(keep_start, 4) || !aligned(keep, 4)) return KVC_ERR_ARG;
    launch_cache_keep(types_of(plan->config), c, keep_start, keep, (int)keep_rows, batch->n, (hipStream_t)hip_stream);
    return hipGetLastError() == hipSuccess ? KVC_OK : KVC_ERR_DEVICE;
}

extern "C" int kvc_cache_attend(const kvc_cache_plan_t *plan, const kvc_cache_batch *batch, const kvc_cache_queries *queries,
                                const void *pages, int32_t *dev_status, void *workspace, void *hip_stream)
{
    using namespace kvc;
    if (!queries) return KVC_ERR_ARG;
    const kvc_cache_queries &u = *queries;
    AttendArgs a;
    const int rc = check_call(plan, batch, (void *)pages, dev_status, u.rows, plan ? plan->max_new : 0, &a.c);
    if (rc != KVC_OK || nothing(batch)) return rc;
    if ((u.rows && (!u.q || !u.out)) || !aligned(u.q, 16) || !aligned(u.out, 16) || !aligned(u.lse, 4) || !strides_ok(u.q_stride_row, u.q_stride_head) ||
        !strides_ok(u.out_stride_row, u.out_stride_head) || !(u.scale >= -3.0e38f && u.scale <= 3.0e38f)) return KVC_ERR_ARG;
    const kvc_cache_config &f = plan->config;
    const AttendShape s = attend_shape(f, batch->n, a.c.max_new, batch->max_tokens);
    if (s.places > kMostThreads / kMostAttending) return KVC_ERR_CAPACITY;
    a.part = a.part_ml = nullptr;
    a.counters = nullptr;
    a.part_rows = 0;
    if (s.divide) {
        const size_t rows = (size_t)s.slots * 16 * s.tiles;
        if (rows * kPartBytes + (size_t)kCounters * sizeof(int) > plan->workspace) return KVC_ERR_CAPACITY;
        if (!workspace || !aligned(workspace, 16)) return KVC_ERR_ARG;
        a.counters = (int *)workspace;
        a.part = (float *)(a.counters + kCounters);
        a.part_ml = a.part + rows * kDim;
        a.part_rows = (long long)rows;
    }
    a.q = (const uint16_t *)u.q;
    a.out = (uint16_t *)u.out;
    a.lse = u.lse;
    a.q_row = u.q_stride_row;
    a.q_head = u.q_stride_head;
    a.o_row = u.out_stride_row;
    a.o_head = u.out_stride_head;
    a.scale = u.scale;
    a.per_kv = f.q_heads / f.kv_heads;
    a.row_blocks = s.row_blocks;
    a.n = batch->n;
    a.divide = s.divide;
    a.parts = (int)s.parts;
    a.joining_piece = s.tiles == kWideTiles ? kManyJoiningPiece : kFewJoiningPiece * s.tiles;
    a.alone = s.tiles == kWideTiles ? kManyAlone : 0.0f;
    a.joining = s.tiles == kWideTiles ? kManyJoining : kFewJoining;
    a.dtype = f.dtype;
    a.rotate = f.transform == KVC_T_HADAMARD;
    const CacheTypes t = types_of(f);
    const hipStream_t stream = (hipStream_t)hip_stream;
    if (f.bits_k == 4 && f.bits_v == 4) launch_attend<44>(t, a, s.tiles, (int)s.places, stream);
    else if (f.bits_k == 4) launch_attend<48>(t, a, s.tiles, (int)s.places, stream);
    else if (f.bits_v == 4) launch_attend<84>(t, a, s.tiles, (int)s.places, stream);
    else launch_attend<88>(t, a, s.tiles, (int)s.places, stream);
    return hipGetLastError() == hipSuccess ? KVC_OK : KVC_ERR_DEVICE;
}
