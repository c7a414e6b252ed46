// Rows of the quantised cache: quantised as they are written, read back, moved.
//
// All three are bound by HBM where there are many rows, and by the latency of a few dependent loads (lengths, page, rows) where there are
// few.  A wave has one granule (16 tokens) of one head, 16 lanes per row and 8 channels per lane, four rows at a time: a group's
// minimum and maximum are found inside a row of lanes, a rotation too, and all of a granule's rows are requested at once.  The
// four waves of a workgroup take neighbouring heads, whose rows lie next to each other in the caller's tensors.
#include "kvc_cache.h"
#include "kvc_cache_internal.h"
#include "../../include/kvc.h"

namespace kvc {

// The lane's 8 values in 32 bits, LIMIT: limited to what scales and zeros can hold, and NaN as 0.
template <int DT, bool LIMIT> __device__ __forceinline__ void values_of(const u32x4 &r, float x[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        x[e] = elem_f32<DT>(r, e);
        if (LIMIT) x[e] = __builtin_amdgcn_fmed3f(x[e] == x[e] ? x[e] : 0.0f, -kTopF16, kTopF16);
    }
}
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
// Whether one of 8 values has to be limited: magnitudes, two at a time, against 65504 or the bf16 number below it.
template <int DT> __device__ __forceinline__ bool out_of_order(const u32x4 &r)
{
    u16x2 m = {0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, (uint32_t)(r[w] & 0x7fff7fffu)));
    constexpr unsigned short most = DT == DT_F16 ? 0x7bff : 0x477f;
    return m[0] > most || m[1] > most;
}

// Codes and parameters of the lane's octet; the parameters are those of the octet's group.
template <int DT, int BITS, int GROUP> __device__ __forceinline__ u32x2 quantise_octet(const float x[8], uint32_t &meta)
{
    float mn = x[0], mx = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        mn = fminf(mn, x[e]);
        mx = fmaxf(mx, x[e]);
    }
    group_minmax<GROUP / 8>(mn, mx);
    const GroupParams g = make_group<BITS, DT>(mn, mx);
    meta = g.meta;
    float t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = (x[e] - g.zero) * g.inv;
    if (__any(g.clamp)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = __builtin_amdgcn_fmed3f(t[e], 0.0f, (float)((1 << BITS) - 1));
    }
    return codes8<BITS, false>(t);
}

// The rows of a granule that are there (from first to before end), to `out`.
template <int DT, int BITS_K, int BITS_V, int GROUP, bool LIMIT>
__device__ __forceinline__ void store_granule(const u32x4 rk[4], const u32x4 rv[4], int col, int first, int end, uint8_t *out)
{
    constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
    constexpr int groups = kDim / GROUP;
    const int rsub = lane_id() >> 4;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int t = 4 * p + rsub;
        if (4 * p + 4 <= first || 4 * p >= end) continue;    // (the same in all lanes: a single row is a quarter of the work)
        float x[8];
        uint32_t mk, mv;
        values_of<DT, LIMIT>(rk[p], x);
        const u32x2 ck = quantise_octet<DT, BITS_K, GROUP>(x, mk);
        values_of<DT, LIMIT>(rv[p], x);
        const u32x2 cv = quantise_octet<DT, BITS_V, GROUP>(x, mv);
        if (t >= first && t < end) {
            if (BITS_K == 4) *(uint32_t *)(out + k_code_at<4>(t, col)) = ck[0];
            else *(u32x2 *)(out + k_code_at<8>(t, col)) = ck;
            uint8_t *tv = out + map.v_codes + v_code_at(t, col);
            *(uint32_t *)tv = cv[0];
            if (BITS_V == 8) *(uint32_t *)(tv + 1024) = cv[1];
            if (col % (GROUP / 8) == 0) {
                const int g = col / (GROUP / 8);
                *(uint16_t *)(out + map.k_scales + k_scale_at<groups>(t, g)) = (uint16_t)mk;
                *(uint16_t *)(out + map.k_zeros + k_zero_at<groups>(t, g)) = (uint16_t)(mk >> 16);
                *(uint16_t *)(out + map.v_params + v_param_at<groups>(t, g)) = (uint16_t)mv;
                *(uint16_t *)(out + map.v_params + v_param_at<groups>(t, g) + 8) = (uint16_t)(mv >> 16);
            }
        }
    }
}

// zero = fp16(min), scale = fp16((max - min) / (2^b - 1)), code = clamp(rint((x - zero) / scale)) per row and group.
// 32k tokens of 8 heads, 4 bits, groups of 32 (134 MB read, 42 written): 41.6 us, 4.2 TB/s (a large copy: 4.8), K rotated 48.
// One token of each of 32 sequences: 3.9 us.
template <int BITS_K, int BITS_V, int GROUP, int DT, bool ROTATE>
__global__ __launch_bounds__(256) void cache_store_kernel(CacheView c, const uint16_t *k, const uint16_t *v, long long stride_row,
                                                          long long stride_head)
{
    constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
    __shared__ __attribute__((aligned(16))) uint8_t space[4][map.bytes];
    const int s = blockIdx.z, quads = (c.heads + 3) >> 2;
    const Sequence seq = sequence_of(c, s);
    const int head = (int)(blockIdx.x % quads) * 4 + wave_id();
    const int past = seq.tokens - seq.fresh;
    const long long j = (past >> 4) + (long long)(blockIdx.x / quads);
    if (seq.fresh == 0 || head >= c.heads || j * kGranule >= seq.tokens) return;
    // (the rotation's lanes hold their octets in an order of their own; V then takes the same order)
    const int col = lane_octet(ROTATE), rsub = lane_id() >> 4;
    u32x4 rk[4], rv[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const long long t = j * kGranule + 4 * p + rsub;
        const bool there = t >= past && t < seq.tokens;
        const long long at = (seq.row0 + (t - past)) * stride_row + head * stride_head + col * 8;
        rk[p] = rv[p] = u32x4{0, 0, 0, 0};
        if (there) {
            rk[p] = __builtin_nontemporal_load((const u32x4 *)(k + at));
            rv[p] = __builtin_nontemporal_load((const u32x4 *)(v + at));
        }
    }
    const int page = __builtin_amdgcn_readfirstlane(page_of(c, s, j));        // (behind the rows' requests)
    if (page < 0) {
        if (lane_id() == 0) atomicOr(c.status + s, KVC_DEV_BAD_BLOCK);
        return;
    }
    uint8_t *to = c.pages + granule_at(c, page, j, head, map.bytes);
    const long long token = j * kGranule;
    const int first = token < past ? (int)(past - token) : 0, end = seq.tokens - token < kGranule ? (int)(seq.tokens - token) : kGranule;
    bool limit = false;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        if (4 * p + 4 <= first || 4 * p >= end) continue;
        // (not limited by the rotation, which would make a number of NaN: rows with values to be limited are found here)
        if (ROTATE) rk[p] = hadamard_row<DT, false>(rk[p], false);
        limit |= out_of_order<DT>(rk[p]) || out_of_order<DT>(rv[p]);
    }
    // A whole granule goes through LDS and out in pieces of 16 bytes per lane, past the caches as its rows came; part of one, and rows
    // with values to be limited, row by row, the parameters two bytes at a time.  (32k tokens of 8 heads, 176 MB: 41.6 us, through the
    // caches 44.8; rotated 48.1 and 51.8.)
    if (first == 0 && end == kGranule && !__any(limit)) {
        uint8_t *own = space[wave_id()];
        store_granule<DT, BITS_K, BITS_V, GROUP, false>(rk, rv, col, 0, kGranule, own);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int at = 0; at < map.bytes; at += 1024) {
            const int mine = at + lane_id() * 16;
            if (mine < map.bytes) put_at<true>(to + mine, *(const u32x4 *)(own + mine));
        }
    } else store_granule<DT, BITS_K, BITS_V, GROUP, true>(rk, rv, col, first, end, to);
}

// Eight codes as numbers: code * scale + zero, one rounding.
template <int BITS> __device__ __forceinline__ void restore_octet(u32x2 w, float scale, float zero, float x[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t code = BITS == 4 ? (w[0] >> (4 * e)) & 15u : (w[e >> 2] >> (8 * (e & 3))) & 255u;
        x[e] = __builtin_fmaf((float)code, scale, zero);
    }
}

template <int DT> __device__ __forceinline__ u32x4 rounded_octet(const float x[8])
{
    u32x4 out;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        f32x2_t v = {__builtin_amdgcn_fmed3f(x[2 * w], -kTopF16, kTopF16), __builtin_amdgcn_fmed3f(x[2 * w + 1], -kTopF16, kTopF16)};
        if (DT == DT_F16) out[w] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
        else out[w] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
    }
    return out;
}

// code * scale + zero in 32 bits, a rotated row turned back, rounded once.  32k tokens of 8 heads, 4 bits, groups of 32, K rotated (42 MB
// read, 134 written): 38 to 43 us, 4.1 to 4.6 TB/s; four sequences of 16k to 32k tokens of 4 heads, 8-bit K, groups of 64 (302 MB): 61.7 us,
// 4.9 TB/s (a large copy: 4.8).  1k tokens of 8 heads: 4.7 us.
template <int BITS_K, int BITS_V, int GROUP, int DT, bool ROTATE>
__global__ __launch_bounds__(256) void cache_load_kernel(CacheView c, uint16_t *k, uint16_t *v, long long stride_row, long long stride_head)
{
    constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
    constexpr int groups = kDim / GROUP;
    const int s = blockIdx.z, quads = (c.heads + 3) >> 2;
    const Sequence seq = sequence_of(c, s);
    const int head = (int)(blockIdx.x % quads) * 4 + wave_id();
    const int past = seq.tokens - seq.fresh;
    const long long j = (past >> 4) + (long long)(blockIdx.x / quads);
    if (seq.fresh == 0 || head >= c.heads || j * kGranule >= seq.tokens) return;
    const int page = __builtin_amdgcn_readfirstlane(page_of(c, s, j));
    if (page < 0) {
        if (lane_id() == 0) atomicOr(c.status + s, KVC_DEV_BAD_BLOCK);
        return;
    }
    const uint8_t *from = c.pages + granule_at(c, page, j, head, map.bytes);
    const int col = lane_id() & 15, rsub = lane_id() >> 4, g = col / (GROUP / 8);
    const long long start = j * kGranule;
    const int first = start < past ? (int)(past - start) : 0, end = seq.tokens - start < kGranule ? (int)(seq.tokens - start) : kGranule;
    u32x2 ck[4], cv[4];
    uint32_t sk[4], zk[4], sv[4], zv[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        if (4 * p + 4 <= first || 4 * p >= end) continue;
        const int t = 4 * p + rsub;              // (rows that nobody wrote are read as well, and not used)
        if (BITS_K == 4) ck[p] = u32x2{*(const uint32_t *)(from + k_code_at<4>(t, col)), 0};
        else ck[p] = *(const u32x2 *)(from + k_code_at<8>(t, col));
        const uint8_t *fv = from + map.v_codes + v_code_at(t, col);
        cv[p] = u32x2{*(const uint32_t *)fv, BITS_V == 8 ? *(const uint32_t *)(fv + 1024) : 0};
        sk[p] = *(const uint16_t *)(from + map.k_scales + k_scale_at<groups>(t, g));
        zk[p] = *(const uint16_t *)(from + map.k_zeros + k_zero_at<groups>(t, g));
        sv[p] = *(const uint16_t *)(from + map.v_params + v_param_at<groups>(t, g));
        zv[p] = *(const uint16_t *)(from + map.v_params + v_param_at<groups>(t, g) + 8);
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        if (4 * p + 4 <= first || 4 * p >= end) continue;
        const long long token = j * kGranule + 4 * p + rsub;
        float x[8], y[8];
        restore_octet<BITS_K>(ck[p], f16_bits_to_f32(sk[p]), f16_bits_to_f32(zk[p]), x);
        if (ROTATE) rotate_row_f32(x, 0.0625f);
        restore_octet<BITS_V>(cv[p], f16_bits_to_f32(sv[p]), f16_bits_to_f32(zv[p]), y);
        if (token >= past && token < seq.tokens) {
            const long long at = (seq.row0 + (token - past)) * stride_row + head * stride_head + col * 8;
            *(u32x4 *)(k + at) = rounded_octet<DT>(x);
            *(u32x4 *)(v + at) = rounded_octet<DT>(y);
        }
    }
}

// Row keep[i] of a sequence's new rows moves to place i.  The indices ascend, so place i is never behind its source: of every 16
// rows all are read before the first is written, and what later rows come from is behind everything written so far.  A wave has
// one head; nothing is decoded.  A few rows per sequence, so latency bounds it (indices, pages, rows, one after the other): 32 sequences
// of 17 to 32 drafts 4.9 us, one of 15 3.7 us.
template <int BITS_K, int BITS_V, int GROUP>
__global__ __launch_bounds__(256) void cache_keep_kernel(CacheView c, const int *keep_start, const int *keep, int max_keep)
{
    constexpr GranuleMap map = granule_map(BITS_K, BITS_V, GROUP);
    constexpr int groups = kDim / GROUP;
    const int s = blockIdx.z, head = (int)blockIdx.x * 4 + wave_id();
    const Sequence seq = sequence_of(c, s);
    const int first = __builtin_amdgcn_readfirstlane(keep_start[s]);
    const int count = __builtin_amdgcn_readfirstlane(keep_start[s + 1]) - first;
    const int past = seq.tokens - seq.fresh;
    const int col = lane_id() & 15, rsub = lane_id() >> 4, g = col;
    if (seq.fresh == 0 && count == 0) return;
    bool bad = first < 0 || (unsigned)count > (unsigned)seq.fresh || (long long)first + count > max_keep;
    if (!bad) {
        for (int i = lane_id(); i < count; i += 64) {
            const int at = keep[first + i], before = i ? keep[first + i - 1] : -1;
            bad |= at <= before || (unsigned)at >= (unsigned)seq.fresh;
        }
    }
    if (__any(bad)) {
        if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(c.status + s, KVC_DEV_BAD_ROW);
        return;                                  // (the same in all waves of the sequence)
    }
    for (int base = 0; base < count; base += 16) {
        u32x2 ck[4], cv[4];
        uint16_t sk[4], zk[4], sv[4], zv[4];
        uint8_t *to[4];
        int slot[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int i = base + 4 * p + rsub;
            to[p] = nullptr;
            slot[p] = 0;
            if (i >= count || head >= c.heads) continue;
            const long long from = past + keep[first + i], dest = past + i;
            const int page = page_of(c, s, from >> 4), page_to = page_of(c, s, dest >> 4);
            if (page < 0 || page_to < 0) {
                atomicOr(c.status + s, KVC_DEV_BAD_BLOCK);
                continue;
            }
            if (from == dest) continue;
            const uint8_t *r = c.pages + granule_at(c, page, from >> 4, head, map.bytes);
            const int t = (int)(from & 15);
            to[p] = c.pages + granule_at(c, page_to, dest >> 4, head, map.bytes);
            slot[p] = (int)(dest & 15);
            if (BITS_K == 4) ck[p] = u32x2{*(const uint32_t *)(r + k_code_at<4>(t, col)), 0};
            else ck[p] = *(const u32x2 *)(r + k_code_at<8>(t, col));
            const uint8_t *rv = r + map.v_codes + v_code_at(t, col);
            cv[p] = u32x2{*(const uint32_t *)rv, BITS_V == 8 ? *(const uint32_t *)(rv + 1024) : 0};
            if (g < groups) {
                sk[p] = *(const uint16_t *)(r + map.k_scales + k_scale_at<groups>(t, g));
                zk[p] = *(const uint16_t *)(r + map.k_zeros + k_zero_at<groups>(t, g));
                sv[p] = *(const uint16_t *)(r + map.v_params + v_param_at<groups>(t, g));
                zv[p] = *(const uint16_t *)(r + map.v_params + v_param_at<groups>(t, g) + 8);
            }
        }
        __syncthreads();
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if (!to[p]) continue;
            const int t = slot[p];
            if (BITS_K == 4) *(uint32_t *)(to[p] + k_code_at<4>(t, col)) = ck[p][0];
            else *(u32x2 *)(to[p] + k_code_at<8>(t, col)) = ck[p];
            uint8_t *tv = to[p] + map.v_codes + v_code_at(t, col);
            *(uint32_t *)tv = cv[p][0];
            if (BITS_V == 8) *(uint32_t *)(tv + 1024) = cv[p][1];
            if (g < groups) {
                *(uint16_t *)(to[p] + map.k_scales + k_scale_at<groups>(t, g)) = sk[p];
                *(uint16_t *)(to[p] + map.k_zeros + k_zero_at<groups>(t, g)) = zk[p];
                *(uint16_t *)(to[p] + map.v_params + v_param_at<groups>(t, g)) = sv[p];
                *(uint16_t *)(to[p] + map.v_params + v_param_at<groups>(t, g) + 8) = zv[p];
            }
        }
        __syncthreads();
    }
}

// ---- launches ---------------------------------------------------------------------------------------

// calls f with the types of a plan as constants
template <typename F> static void with_store_types(const CacheTypes &t, F f)
{
    auto by_group = [&](auto bk, auto bv) {
        if (t.group == 32) f(bk, bv, IntConst<32>());
        else if (t.group == 64) f(bk, bv, IntConst<64>());
        else f(bk, bv, IntConst<128>());
    };
    if (t.bits_k == 4 && t.bits_v == 4) by_group(IntConst<4>(), IntConst<4>());
    else if (t.bits_k == 4) by_group(IntConst<4>(), IntConst<8>());
    else if (t.bits_v == 4) by_group(IntConst<8>(), IntConst<4>());
    else by_group(IntConst<8>(), IntConst<8>());
}

// granules that max_new consecutive tokens can lie in, by four heads
long long row_places(const CacheView &c) { return ((long long)c.max_new + 2 * kGranule - 2) / kGranule * ((c.heads + 3) / 4); }

void launch_cache_rows(const CacheTypes &t, const CacheView &c, bool store, uint16_t *k, uint16_t *v, long long stride_row,
                       long long stride_head, int n, hipStream_t stream)
{
    const dim3 grid((unsigned)row_places(c), 1, (unsigned)n);
    with_store_types(t, [&](auto bk, auto bv, auto g) {
        constexpr int BK = decltype(bk)::value, BV = decltype(bv)::value, G = decltype(g)::value;
        auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, c, k, v, stride_row, stride_head); };
        if (store) {
            if (t.dtype == DT_F16) {
                if (t.rotate) run(cache_store_kernel<BK, BV, G, DT_F16, true>);
                else run(cache_store_kernel<BK, BV, G, DT_F16, false>);
            } else {
                if (t.rotate) run(cache_store_kernel<BK, BV, G, DT_BF16, true>);
                else run(cache_store_kernel<BK, BV, G, DT_BF16, false>);
            }
        } else {
            if (t.dtype == DT_F16) {
                if (t.rotate) run(cache_load_kernel<BK, BV, G, DT_F16, true>);
                else run(cache_load_kernel<BK, BV, G, DT_F16, false>);
            } else {
                if (t.rotate) run(cache_load_kernel<BK, BV, G, DT_BF16, true>);
                else run(cache_load_kernel<BK, BV, G, DT_BF16, false>);
            }
        }
    });
}

void launch_cache_keep(const CacheTypes &t, const CacheView &c, const int *keep_start, const int *keep, int max_keep, int n,
                       hipStream_t stream)
{
    const dim3 grid((unsigned)((c.heads + 3) / 4), 1, (unsigned)n);
    with_store_types(t, [&](auto bk, auto bv, auto g) {
        hipLaunchKernelGGL((cache_keep_kernel<decltype(bk)::value, decltype(bv)::value, decltype(g)::value>), grid, dim3(256), 0, stream,
                           c, keep_start, keep, max_keep);
    });
}

}  // namespace kvc
