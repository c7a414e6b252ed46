// Host side of the calls on prompts: plans, frequencies of the rotation, checks of the arguments.
#include "kvc_prompt_internal.h"
#include "../../include/kvc.h"

#include <math.h>
#include <new>

struct kvc_prompt_plan_s {
    kvc_prompt_config config;
    int32_t max_batch;
    uint64_t turns[kvc::kMostPairs];
};

namespace kvc {

constexpr double kTwoPi = 6.283185307179586;

constexpr int64_t kMostStride = 1 << 24;      // of rows of K and V, in elements
constexpr int64_t kMostRows = 1 << 28;        // of a call
constexpr int64_t kMostThreads = 0xffffffffll;       // of a launch

static bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
static bool strides_ok(int64_t row, int64_t head) { return row % 8 == 0 && head % 8 == 0; }
// Results apart from the input, or in its place.
static bool in_place_ok(const void *in, const void *out, int64_t rows, int64_t heads, int64_t row, int64_t head, int64_t out_row, int64_t out_head)
{
    return in != out || ((rows < 2 || row == out_row) && (heads < 2 || head == out_head));
}

// 1 / (2 pi) in 2^-128
constexpr unsigned __int128 kTurnsPerRadian = (unsigned __int128)0x28be60db9391054aull << 64 | 0x7f09d5f47d4d3770ull;

// Heads of a result that lie apart: rows * row + heads * head comes nowhere within a head of itself.  (Two that share a place would race for it.)
static bool apart(int64_t rows, int64_t heads, int64_t row, int64_t head)
{
    if (rows < 1) return true;
    typedef __int128 wide;                   // (strides are any 64-bit numbers)
    const wide r = row < 0 ? -(wide)row : row, h = head < 0 ? -(wide)head : head;
    if ((rows > 1 && r < kDim) || (heads > 1 && h < kDim)) return false;
    if (rows < 2 || heads < 2 || r >= (heads - 1) * h + kDim || h >= (rows - 1) * r + kDim) return true;
    for (wide d = 1; d < heads; ++d) {       // (only layouts that are neither rows of heads nor heads of rows)
        const wide below = d * h / r, off = d * h - below * r;
        if ((below < rows && off < kDim) || (below + 1 < rows && r - off < kDim)) return false;
    }
    return true;
}

// The part of a turn that a position adds, in 2^-64 of a turn, rounded.  The product is made of whole numbers: of a frequency of 10^9 radians the turns
// that are dropped have 28 bits, which a floating-point quotient would have in place of the last ones that a large position needs.
static uint64_t turns_of(double radians)
{
    int exponent;
    const uint64_t mantissa = (uint64_t)ldexp(frexp(fabs(radians), &exponent), 53);       // times 2^(exponent - 53)
    const unsigned __int128 low = (unsigned __int128)mantissa * (uint64_t)kTurnsPerRadian;
    const unsigned __int128 high = (unsigned __int128)mantissa * (uint64_t)(kTurnsPerRadian >> 64) + (uint64_t)(low >> 64);       // in 2^(exponent - 117)
    const int down = 53 - exponent;          // to 2^-64: 23 at least, since frequencies are no more than 10^9
    if (down > 127) return 0;
    const uint64_t turns = (uint64_t)(high >> down) + (uint64_t)(high >> (down - 1) & 1);
    return radians < 0 ? 0 - turns : turns;
}

}  // namespace kvc

extern "C" int kvc_rotary_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double low, double high,
                                      int64_t original_tokens, double *frequencies)
{
    if (!frequencies || rotary_dim < 2 || rotary_dim % 2 || !(base > 1.0) || !(base <= 1e300)) return KVC_ERR_ARG;
    if (scaling < KVC_SCALE_NONE || scaling > KVC_SCALE_RAMP) return KVC_ERR_ARG;
    if (scaling != KVC_SCALE_NONE && !(factor >= 1.0 && factor <= 1e9)) return KVC_ERR_ARG;
    const bool windows = scaling == KVC_SCALE_BANDS || scaling == KVC_SCALE_RAMP;
    if (windows && (!(low > 0.0) || !(high > low) || !(high <= 1e9) || original_tokens < 1)) return KVC_ERR_ARG;
    if (scaling == KVC_SCALE_BASE && rotary_dim == 2) return KVC_ERR_ARG;
    const double R = rotary_dim, two_pi = kvc::kTwoPi, original = (double)original_tokens;
    if (scaling == KVC_SCALE_BASE) base *= pow(factor, R / (R - 2.0));
    double first = 0.0, last = 0.0;
    if (scaling == KVC_SCALE_RAMP) {
        first = floor(R * log(original / (high * two_pi)) / (2.0 * log(base)));
        last = ceil(R * log(original / (low * two_pi)) / (2.0 * log(base)));
        first = first > 0.0 ? first : 0.0;
        last = last < R - 1.0 ? last : R - 1.0;
    }
    for (int32_t i = 0; i < rotary_dim / 2; ++i) {
        const double f = pow(base, -2.0 * i / R);
        double t = 1.0;                                  // the share of the unscaled frequency
        if (scaling == KVC_SCALE_LINEAR) t = 0.0;
        else if (scaling == KVC_SCALE_BANDS) t = (original * f / two_pi - low) / (high - low);
        else if (scaling == KVC_SCALE_RAMP) t = 1.0 - (i - first) / (last - first > 0.001 ? last - first : 0.001);
        t = t < 0.0 ? 0.0 : t > 1.0 ? 1.0 : t;
        frequencies[i] = scaling == KVC_SCALE_NONE || scaling == KVC_SCALE_BASE ? f : t * f + (1.0 - t) * f / factor;
    }
    return KVC_OK;
}

extern "C" int kvc_prompt_plan(const kvc_prompt_config *config, int32_t max_batch, kvc_prompt_plan_t **out)
{
    using namespace kvc;
    if (!out) return KVC_ERR_ARG;
    *out = nullptr;
    if (!config || max_batch < 1) return KVC_ERR_ARG;
    const kvc_prompt_config &f = *config;
    if (f.dtype != KVC_F16 && f.dtype != KVC_BF16) return KVC_ERR_ARG;
    if (f.norm > 1 || (f.layout != KVC_ROTARY_HALVES && f.layout != KVC_ROTARY_PAIRS)) return KVC_ERR_ARG;
    if (f.kv_heads < 1 || f.q_heads < 1 || f.q_heads % f.kv_heads || f.head_dim < 1) return KVC_ERR_ARG;
    if (f.rotary_dim < 0 || f.rotary_dim > f.head_dim || f.rotary_dim % 2 || (f.rotary_dim && !f.frequencies)) return KVC_ERR_ARG;
    if (f.norm && !(f.eps >= 0.0f && f.eps <= 1e30f)) return KVC_ERR_ARG;
    if (f.rotary_dim && !(f.amplitude > 0.0f && f.amplitude <= 1e30f)) return KVC_ERR_ARG;
    for (int i = 0; i < f.rotary_dim / 2; ++i)
        if (!(f.frequencies[i] >= -1e9 && f.frequencies[i] <= 1e9)) return KVC_ERR_ARG;
    if (f.head_dim != kDim || f.rotary_dim % 16 || f.q_heads > 65535 || max_batch > 65535) return KVC_ERR_UNSUPPORTED;
    kvc_prompt_plan_t *p = new (std::nothrow) kvc_prompt_plan_t();
    if (!p) return KVC_ERR_CAPACITY;
    p->config = f;
    p->config.frequencies = nullptr;
    p->max_batch = max_batch;
    for (int i = 0; i < f.rotary_dim / 2; ++i) p->turns[i] = turns_of(f.frequencies[i]);
    *out = p;
    return KVC_OK;
}

extern "C" void kvc_prompt_plan_free(kvc_prompt_plan_t *plan) { delete plan; }

extern "C" int kvc_prompt_rotate(const kvc_prompt_plan_t *plan, const kvc_prompt_rows *r, void *hip_stream)
{
    using namespace kvc;
    if (!plan || !r || r->rows < 0) return KVC_ERR_ARG;
    const kvc_prompt_config &f = plan->config;
    if (r->rows == 0 || (!r->q && !r->k)) return KVC_OK;
    if ((r->q && !r->q_out) || (r->k && !r->k_out) || (f.norm && ((r->q && !r->q_weight) || (r->k && !r->k_weight)))) return KVC_ERR_ARG;
    if (f.rotary_dim && !r->positions) return KVC_ERR_ARG;
    if (!aligned(r->q, 16) || !aligned(r->k, 16) || !aligned(r->q_out, 16) || !aligned(r->k_out, 16) || !aligned(r->q_weight, 16) ||
        !aligned(r->k_weight, 16) || !aligned(r->positions, 4)) return KVC_ERR_ARG;
    if (!strides_ok(r->q_stride_row, r->q_stride_head) || !strides_ok(r->k_stride_row, r->k_stride_head) ||
        !strides_ok(r->q_out_stride_row, r->q_out_stride_head) || !strides_ok(r->k_out_stride_row, r->k_out_stride_head)) return KVC_ERR_ARG;
    if ((r->q && (!in_place_ok(r->q, r->q_out, r->rows, f.q_heads, r->q_stride_row, r->q_stride_head, r->q_out_stride_row, r->q_out_stride_head) ||
                  r->q_out == r->k)) ||
        (r->k && (!in_place_ok(r->k, r->k_out, r->rows, f.kv_heads, r->k_stride_row, r->k_stride_head, r->k_out_stride_row, r->k_out_stride_head) ||
                  r->k_out == r->q)) || (r->q && r->k && r->q_out == r->k_out)) return KVC_ERR_ARG;
    if (r->rows > kMostRows) return KVC_ERR_CAPACITY;
    if ((r->q && !apart(r->rows, f.q_heads, r->q_out_stride_row, r->q_out_stride_head)) ||
        (r->k && !apart(r->rows, f.kv_heads, r->k_out_stride_row, r->k_out_stride_head))) return KVC_ERR_ARG;
    RotateArgs a = {};
    a.q = RotateTensor{(const uint16_t *)r->q, f.norm ? (const uint16_t *)r->q_weight : nullptr, (uint16_t *)r->q_out, r->q_stride_row,
                       r->q_stride_head, r->q_out_stride_row, r->q_out_stride_head, r->q ? f.q_heads : 0, 0};
    a.k = RotateTensor{(const uint16_t *)r->k, f.norm ? (const uint16_t *)r->k_weight : nullptr, (uint16_t *)r->k_out, r->k_stride_row,
                       r->k_stride_head, r->k_out_stride_row, r->k_out_stride_head, r->k ? f.kv_heads : 0, 0};
    a.positions = r->positions;
    a.rows = r->rows;
    a.eps = f.eps;
    a.amplitude = f.rotary_dim ? f.amplitude : 1.0f;
    a.pairs = f.rotary_dim / 2;
    for (int i = 0; i < a.pairs; ++i) a.turns[i] = plan->turns[i];
    divide_rows(a);
    // one launch for as many rows as its threads can be (2^26, or 13 million with 64 + 8 heads), further ones behind it
    const int64_t most = kMostThreads / 256 * 4 / a.chunks;
    for (int64_t done = 0; done < r->rows; done += most) {
        RotateArgs part = a;
        part.rows = r->rows - done < most ? r->rows - done : most;
        if (done) {
            for (RotateTensor *x : {&part.q, &part.k}) {
                if (!x->heads) continue;
                x->in += done * x->in_row;
                x->out += done * x->out_row;
            }
            if (part.positions) part.positions += done;
        }
        launch_rotate(f.dtype, f.layout == KVC_ROTARY_PAIRS, f.norm != 0, part, (part.rows * part.chunks + 3) / 4, (hipStream_t)hip_stream);
        if (hipGetLastError() != hipSuccess) return KVC_ERR_DEVICE;
    }
    return KVC_OK;
}

extern "C" int32_t kvc_prompt_block_rows(const kvc_prompt_plan_t *plan, int32_t n, int32_t max_rows, int64_t rows, int32_t *waves)
{
    using namespace kvc;
    if (waves) *waves = 0;
    if (!plan || n < 1 || max_rows < 1 || rows < 1 || n > plan->max_batch || rows > kMostRows) return 0;
    PromptArgs a = {};
    a.n = n;
    a.max_rows = max_rows;
    a.rows = rows;
    a.kv_heads = plan->config.kv_heads;
    a.per_kv = plan->config.q_heads / plan->config.kv_heads;
    int many;
    const int block = prompt_block_rows(a, many);
    if (waves) *waves = many;
    return block;
}

extern "C" int kvc_prompt_attend(const kvc_prompt_plan_t *plan, const kvc_prompt_batch *batch, const kvc_prompt_heads *heads,
                                 int32_t *dev_status, void *hip_stream)
{
    using namespace kvc;
    if (!plan || !batch || !heads) return KVC_ERR_ARG;
    const kvc_prompt_config &f = plan->config;
    const kvc_prompt_heads &h = *heads;
    if (batch->n < 0 || batch->max_rows < 0 || h.rows < 0) return KVC_ERR_ARG;
    if (batch->n > plan->max_batch || h.rows > kMostRows) return KVC_ERR_CAPACITY;
    if (batch->n == 0 || batch->max_rows == 0) return KVC_OK;
    if (!batch->start || !dev_status || (h.rows && (!h.q || !h.k || !h.v || !h.out))) return KVC_ERR_ARG;
    if (!aligned(batch->start, 4) || !aligned(dev_status, 4) || !aligned(h.q, 16) || !aligned(h.k, 16) || !aligned(h.v, 16) || !aligned(h.out, 16) ||
        !aligned(h.lse, 4)) return KVC_ERR_ARG;
    if (!strides_ok(h.q_stride_row, h.q_stride_head) || !strides_ok(h.k_stride_row, h.k_stride_head) ||
        !strides_ok(h.v_stride_row, h.v_stride_head) || !strides_ok(h.out_stride_row, h.out_stride_head)) return KVC_ERR_ARG;
    if (h.out && (h.out == h.k || h.out == h.v ||
                  !in_place_ok(h.q, h.out, h.rows, f.q_heads, h.q_stride_row, h.q_stride_head, h.out_stride_row, h.out_stride_head))) return KVC_ERR_ARG;
    if (!apart(h.rows, f.q_heads, h.out_stride_row, h.out_stride_head)) return KVC_ERR_ARG;
    // (smaller factors are subnormal numbers, which may count as zero)
    if (!(fabsf(h.scale) <= 1e38f) || (h.scale != 0.0f && fabsf(h.scale) < 1e-37f)) return KVC_ERR_ARG;
    // (offsets of the 64 rows of a tile are 32-bit numbers above zero)
    if (h.k_stride_row < 0 || h.v_stride_row < 0 || h.k_stride_row > kMostStride || h.v_stride_row > kMostStride) return KVC_ERR_UNSUPPORTED;
    PromptArgs a = {};
    a.q = (const uint16_t *)h.q;
    a.k = (const uint16_t *)h.k;
    a.v = (const uint16_t *)h.v;
    a.out = (uint16_t *)h.out;
    a.lse = h.lse;
    a.start = batch->start;
    a.status = dev_status;
    a.rows = h.rows;
    a.q_row = h.q_stride_row, a.q_head = h.q_stride_head;
    a.k_row = h.k_stride_row, a.k_head = h.k_stride_head;
    a.v_row = h.v_stride_row, a.v_head = h.v_stride_head;
    a.o_row = h.out_stride_row, a.o_head = h.out_stride_head;
    // (a factor of zero would turn the -infinity of scores that are not seen into NaN)
    a.factor = h.scale == 0.0f ? 1.0f : fabsf(h.scale) * 1.44269504f;
    a.query_and = h.scale == 0.0f ? 0u : 0xffffffffu;
    a.query_xor = h.scale < 0.0f ? 0x80008000u : 0u;
    a.n = batch->n;
    a.max_rows = batch->max_rows;
    a.kv_heads = f.kv_heads;
    a.per_kv = f.q_heads / f.kv_heads;
    launch_prompt(f.dtype, a, (hipStream_t)hip_stream);
    return hipGetLastError() == hipSuccess ? KVC_OK : KVC_ERR_DEVICE;
}
