// Queries and keys of new rows: every head normed and rotated by the row's position, in one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * w          (where the plan norms heads)
//   (a, b) <- A (a cos t - b sin t, a sin t + b cos t),   t = position * frequency of the pair
//
// All in 32 bits, rounded once as it is stored.  Bound by HBM where there are many rows (every element is read and written once) and by
// latency where there are few.  A wave has one row and a run of its heads, four heads at a time, 16 lanes per head and 8 channels
// per lane: cosines and sines are made once per row and wave, the mean of a head inside a row of lanes.  32k rows of 72 heads: 192 to 198 us, 6.1 to 6.3 TB/s
// (cards differ; the fastest copy found 6.5); 32 rows 3.3 us in a graph, most of it the launch.
//
// Angles are fixed-point numbers of 2^-64 of a turn: a position times a frequency's part of a turn, modulo a turn, is one integer product
// whose upper word is the angle, exact to 2^-32 of a turn wherever the position is (in 32-bit floating point a position of 10^6 would be
// off by 0.03 radians).  Sine and cosine are the Taylor polynomials of degree 9 and 8 on an eighth of a turn to either side of a
// quarter's multiple (the first terms left out: 2e-9 and 3e-8).
#include "kvc_prompt_internal.h"

namespace kvc {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int DT> __device__ __forceinline__ uint32_t round_pair(float a, float b)
{
    const f32x2 x = {a, b};
    if constexpr (DT == DT_F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// cos and sin of t * 2^-32 turns
__device__ __forceinline__ void turn(uint32_t t, float &c, float &s)
{
    const uint32_t quarter = (t + 0x20000000u) >> 30;
    const float x = (float)(int)(t - (quarter << 30)) * 1.46291807926715968e-9f;       // 2 pi / 2^32
    const float y = x * x;
    float sine = __builtin_fmaf(y, 2.75573192e-6f, -1.98412698e-4f);
    sine = __builtin_fmaf(y, sine, 8.33333333e-3f);
    sine = __builtin_fmaf(y, sine, -1.66666667e-1f);
    sine = __builtin_fmaf(x * y, sine, x);
    float cosine = __builtin_fmaf(y, 2.48015873e-5f, -1.38888889e-3f);
    cosine = __builtin_fmaf(y, cosine, 4.16666667e-2f);
    cosine = __builtin_fmaf(y, cosine, -0.5f);
    cosine = __builtin_fmaf(y, cosine, 1.0f);
    const bool odd = quarter & 1;
    c = odd ? sine : cosine;
    s = odd ? cosine : sine;
    c = (quarter + 1) & 2 ? -c : c;
    s = quarter & 2 ? -s : s;
}

template <int N> __device__ __forceinline__ float turned_lane(float x)       // the value N lanes further in the row of 16
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x120 + N, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum_of_row(float x)
{
    x += turned_lane<8>(x);
    x += turned_lane<4>(x);
    x += turned_lane<2>(x);
    return x + turned_lane<1>(x);
}

// The octet of channels of the lane that holds the other half of the lane's pairs.
__device__ __forceinline__ u32x4 other_octet(const u32x4 &x, int other, bool opposite)
{
    u32x4 r;
    if (opposite) {                          // all 128 channels in halves: the lane 8 further
#pragma unroll
        for (int w = 0; w < 4; ++w) r[w] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x[w], 0x128, 0xf, 0xf, true);
    } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) r[w] = (uint32_t)__builtin_amdgcn_ds_bpermute(other * 4, (int)x[w]);
    }
    return r;
}

constexpr int kAtOnce = 4;                    // groups of four heads that a wave requests together
template <int N> struct Count {
    static constexpr int value = N;
};

template <int DT, bool NEIGHBOURS, bool NORM> __global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a)
{
    const long long unit = (long long)blockIdx.x * 4 + wave_id();
    const long long row = unit / a.chunks;
    if (row >= a.rows) return;
    const int position = a.positions ? __builtin_amdgcn_readfirstlane(a.positions[row]) : 0;
    if (position < 0) return;
    const int q_chunks = (a.q.heads + a.chunk - 1) / a.chunk;
    const int part = (int)(unit - row * a.chunks);
    const bool is_k = part >= q_chunks;
    const RotateTensor &x = is_k ? a.k : a.q;
    const int first = (is_k ? part - q_chunks : part) * a.chunk;
    const int end = first + a.chunk < x.heads ? first + a.chunk : x.heads;
    const int lane = lane_id(), col = lane & 15, sub = lane >> 4;

    // Factors of the lane's channels and of their partners'.  With norms of bf16 heads the amplitude is left for the head's own factor, and that
    // comes first: a weight times a normed number stays inside 32 bits where the type's numbers times each other do not.
    constexpr bool APART = NORM && DT == DT_BF16;
    float own[8], other[8];
    const int half = a.pairs / 8;            // octets of one half
    const bool turns = col < 2 * half, front = col < half;
    const int partner = NEIGHBOURS || !turns ? lane : front ? lane + half : lane - half;
    if (turns) {
        const uint64_t *f = a.turns + (NEIGHBOURS ? 4 * col : 8 * (front ? col : col - half));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (NEIGHBOURS && (e & 1)) {
                own[e] = own[e - 1];
                other[e] = -other[e - 1];
                continue;
            }
            const uint64_t each = f[NEIGHBOURS ? e / 2 : e];
            float c, s;
            turn(__umulhi((uint32_t)position, (uint32_t)each) + (uint32_t)position * (uint32_t)(each >> 32), c, s);
            own[e] = APART ? c : c * a.amplitude;
            other[e] = APART ? (NEIGHBOURS || front ? -s : s) : (NEIGHBOURS || front ? -s : s) * a.amplitude;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            own[e] = 1.0f;
            other[e] = 0.0f;
        }
    }
    if (NORM) {
        const u32x4 w = *(const u32x4 *)(x.weight + 8 * col);
        const u32x4 p = NEIGHBOURS ? w : other_octet(w, partner, false);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            own[e] *= elem_f32<DT>(w, e);
            other[e] *= elem_f32<DT>(p, NEIGHBOURS ? e ^ 1 : e);
        }
    }
    const uint16_t *in = x.in + row * x.in_row + 8 * col;
    uint16_t *out = x.out + row * x.out_row + 8 * col;
    // GROUPS of four heads at a time, all requested at once
    auto do_heads = [&](int h, auto groups) {
        constexpr int GROUPS = decltype(groups)::value;
        u32x4 r[GROUPS];
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            const int head = h + 4 * u + sub < end ? h + 4 * u + sub : end - 1;
            const u32x4 *from = (const u32x4 *)(in + head * x.in_head);
            r[u] = a.past_caches ? __builtin_nontemporal_load(from) : *from;
        }
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            const int head = h + 4 * u + sub;
            const u32x4 p = NEIGHBOURS ? r[u] : other_octet(r[u], partner, half == 8);
            float mine[8], theirs[8], y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                mine[e] = elem_f32<DT>(r[u], e);
                theirs[e] = elem_f32<DT>(p, NEIGHBOURS ? e ^ 1 : e);
            }
            float by = 1.0f;
            if (NORM) {
                float sum = 0.0f, eps = a.eps;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(mine[e], mine[e], sum);
                sum = sum_of_row(sum);
                // bf16 values whose squares leave 32 bits: all of the head times a power of two
                const bool large = sum > 1e38f, small = sum < 1e-30f && eps < 1e-30f;
                if (DT == DT_BF16 && __any(large || small)) {
                    const float f = large ? 0x1p-70f : small ? 0x1p80f : 1.0f;
                    sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        mine[e] *= f;
                        theirs[e] *= f;
                        sum = __builtin_fmaf(mine[e], mine[e], sum);
                    }
                    sum = sum_of_row(sum);
                    eps = eps * f * f;               // (the square alone may leave 32 bits)
                }
                by = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, 1.0f / kDim, eps));
            }
            if (APART) {
                if (turns) by *= a.amplitude;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    mine[e] *= by;
                    theirs[e] *= by;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = mine[e] * own[e];
                if (turns) y[e] = __builtin_fmaf(theirs[e], other[e], y[e]);
                if (NORM && !APART) y[e] *= by;
            }
            // (Stored past the caches: alone 1k rows of 40 heads take 5.9 instead of 6.8 us, 32k rows of 72 heads 199 instead of 210; what reads them next
            // pays where the caches had held them: 8k rows of 40 heads and their attention as prompts of 512 101 instead of 97, 1k rows 27.0 instead of 28.3.)
            if (head < end) {
                const u32x4 z = {round_pair<DT>(y[0], y[1]), round_pair<DT>(y[2], y[3]), round_pair<DT>(y[4], y[5]), round_pair<DT>(y[6], y[7])};
                __builtin_nontemporal_store(z, (u32x4 *)(out + head * x.out_head));
            }
        }
    };
    int h = first;
    for (; h + 4 * kAtOnce <= end; h += 4 * kAtOnce) do_heads(h, Count<kAtOnce>());
    for (; h < end; h += 4) do_heads(h, Count<1>());
}

template <int DT, bool NEIGHBOURS> static void launch_layout(bool norm, const RotateArgs &a, dim3 grid, hipStream_t stream)
{
    if (norm) rotate_kernel<DT, NEIGHBOURS, true><<<grid, 256, 0, stream>>>(a);
    else rotate_kernel<DT, NEIGHBOURS, false><<<grid, 256, 0, stream>>>(a);
}

// Heads of a row that a wave takes: up to 16, which are 4 KB in a row for each of a workgroup's waves (32k rows of 72 heads: 192 us, with all of a row
// in one wave 214, with 8 heads 225); fewer while there are not that many waves (1k rows of 40 heads: 5.5 us, with waves of 4 heads 7.9).
constexpr int kMostHeads = 16;
constexpr long long kLeastWaves = 4096;
// Bytes read and written beyond which rows are read past the caches, which cannot hold them for anyone (32k rows of 72 heads, 1.2 GB: 192 instead of
// 229 us; 8k rows of 40 heads, 168 MB: 30 instead of 29).
constexpr double kCaches = 256e6;

// How a call's rows are divided.
void divide_rows(RotateArgs &a)
{
    const int most = a.q.heads > a.k.heads ? a.q.heads : a.k.heads;
    auto chunks = [&](int chunk) { return (a.q.heads + chunk - 1) / chunk + (a.k.heads + chunk - 1) / chunk; };
    a.chunk = most < kMostHeads ? (most + 3) / 4 * 4 : kMostHeads;
    while (a.chunk > 4 && a.rows * chunks(a.chunk) < kLeastWaves) a.chunk -= 4;
    a.chunks = chunks(a.chunk);
    a.past_caches = (double)a.rows * (a.q.heads + a.k.heads) * 4 * kDim > kCaches;
}
void launch_rotate(int dtype, bool neighbours, bool norm, const RotateArgs &a, long long groups, hipStream_t stream)
{
    const dim3 grid((unsigned)groups);
    if (dtype == DT_F16) neighbours ? launch_layout<DT_F16, true>(norm, a, grid, stream) : launch_layout<DT_F16, false>(norm, a, grid, stream);
    else neighbours ? launch_layout<DT_BF16, true>(norm, a, grid, stream) : launch_layout<DT_BF16, false>(norm, a, grid, stream);
}

}  // namespace kvc
