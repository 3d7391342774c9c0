// The pages a new token attends to: each page is scored by the largest product
// that the bounds of its keys (smallest and largest per channel) allow with a
// query of the kv head's group,
//
//   score = max_h sum_c (q_hc > 0 ? q_hc hi_c : q_hc lo_c)
//         = max_h (min(q_h, 0) . lo + max(q_h, 0) . hi),
//
// a product over 2 D channels for the MFMAs, and the best `select` are kept in the
// order of their positions.
#include <hip/hip_runtime.h>

#include "kv.h"
#include "kv_device.h"

namespace marlin {
namespace {

using namespace dev;

constexpr int kScoreWaves = 4, kScorePages = 16 * kScoreWaves;

__device__ __forceinline__ int pages_of(const SelectProblem &p, int b)
{
    const int n = p.lengths[b], cap = p.width << p.page_shift;
    const int len = n < 0 ? 0 : n < cap ? n : cap;
    return (len + (1 << p.page_shift) - 1) >> p.page_shift;
}

// fp32 to integers in the same order, all of them from 1 to 2^32 - 3; a score
// that is not a number is 2^32 - 2.
constexpr uint32_t kNoPage = 0u, kNan = 0xFFFFFFFEu, kLastPage = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t score_key(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);  // -0 and 0 are equal
    return x != x ? kNan : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// A wave scores 16 pages: lane (r = l % 16, g = l / 16) loads 16-byte pieces of page
// r's bounds and gets the products of heads 4g .. 4g + 3 with it.
template <typename T, int D>
__global__ void __launch_bounds__(64 * kScoreWaves) page_score_kernel(const SelectProblem p)
{
    typedef typename Elem<T>::vec8 vec8;
    constexpr int kQ = D / 32;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int blocks = (p.width + kScorePages - 1) / kScorePages;
    const int row = blockIdx.x / blocks, b = row / p.kv_heads, kvh = row % p.kv_heads;
    const int pages = pages_of(p, b), page0 = (int)(blockIdx.x % blocks) * kScorePages + wave * 16;
    if (pages <= p.select || page0 >= pages) return;
    const int at = page0 + r;
    const int page = at < pages ? p.table[b * p.table_row + at] : -1;
    const bool inside = (uint32_t)page < (uint32_t)p.pages;
    const T *box = (const T *)p.bounds + ((int64_t)(inside ? page : 0) * p.kv_heads + kvh) * 2 * D + 8 * g;
    vec8 lo[kQ], hi[kQ];
#pragma unroll
    for (int t = 0; t < kQ; ++t) {
        lo[t] = *(const vec8 *)(box + 32 * t);
        hi[t] = *(const vec8 *)(box + D + 32 * t);
    }
    float best = -INFINITY;
    bool nan = false;
    for (int h0 = 0; h0 < p.group; h0 += 16) {
        const T *q = (const T *)p.q + b * p.q_row + (kvh * p.group + h0 + r) * p.q_head + 8 * g;
        float4_t s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < kQ; ++t) {
            const vec8 x = h0 + r < p.group ? *(const vec8 *)(q + 32 * t) : vec8{};
            vec8 neg, pos;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                pos[e] = x[e] > (T)0.f ? x[e] : (T)0.f;
                neg[e] = x[e] > (T)0.f ? (T)0.f : x[e];
            }
            s = Elem<T>::mfma(neg, lo[t], s);
            s = Elem<T>::mfma(pos, hi[t], s);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (h0 + 4 * g + i < p.group) {
                best = fmaxf(best, s[i]);
                nan |= s[i] != s[i];
            }
    }
    best = max_over_groups(best);
    const uint64_t nans = __ballot(nan);
    nan = (nans >> r | nans >> (r + 16) | nans >> (r + 32) | nans >> (r + 48)) & 1;
    if (g == 0 && at < pages)
        p.scores[(int64_t)row * p.width + at] = at == pages - 1 ? kLastPage : !inside ? kNoPage
                                                                   : nan          ? kNan
                                                                                  : score_key(best);
}

// One work-group per (sequence, kv head): the select-th largest score, a byte at a
// time from counts of the candidates' bytes, then every page above it and the
// first ones equal to it, in order.
constexpr int kPickThreads = 512;

__global__ void __launch_bounds__(kPickThreads) page_pick_kernel(const SelectProblem p)
{
    __shared__ int count[256], above, bucket, totals[kPickThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.x / p.kv_heads, kvh = blockIdx.x % p.kv_heads;
    const int pages = pages_of(p, b);
    const int32_t *table = p.table + b * p.table_row;
    int32_t *out = p.chosen + (int64_t)blockIdx.x * p.select;
    if (kvh == 0 && tid == 0) {
        const int n = p.lengths[b], cap = p.width << p.page_shift, len = n < 0 ? 0 : n < cap ? n : cap;
        p.chosen_lengths[b] = pages > p.select ? len - ((pages - p.select) << p.page_shift) : len;
    }
    if (pages <= p.select) {
        for (int i = tid; i < p.select; i += kPickThreads) out[i] = i < pages ? table[i] : -1;
        return;
    }
    const uint32_t *scores = p.scores + (int64_t)blockIdx.x * p.width;
    uint32_t prefix = 0;
    int want = p.select;  // of the candidates, those whose higher bytes are prefix's
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kPickThreads) count[i] = 0;
        __syncthreads();
        for (int i = tid; i < pages; i += kPickThreads) {
            const uint32_t s = scores[i];
            if (shift == 24 || (s >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&count[(s >> shift) & 255], 1);
        }
        __syncthreads();
        if (wave == 0) {
            // lane l: bytes 255 - 4l .. 252 - 4l, from the top
            int c[4], sum = 0;
            for (int k = 0; k < 4; ++k) sum += c[k] = count[255 - 4 * lane - k];
            int upto = wave_scan(sum) - sum;
            for (int k = 0; k < 4; ++k) {
                if (upto < want && want <= upto + c[k]) {
                    bucket = 255 - 4 * lane - k;
                    above = upto;
                }
                upto += c[k];
            }
        }
        __syncthreads();
        prefix |= (uint32_t)bucket << shift;
        want -= above;
    }
    // every score above prefix, and the first `want` equal to it
    int placed = 0, equal = 0;
    for (int i0 = 0; i0 < pages; i0 += kPickThreads) {
        const int i = i0 + tid;
        const uint32_t s = i < pages ? scores[i] : 0;
        const bool same = i < pages && s == prefix;
        const uint64_t sames = __ballot(same);
        const uint64_t below = ((uint64_t)1 << lane) - 1;
        __syncthreads();
        if (lane == 0) totals[wave] = __popcll(sames);
        __syncthreads();
        int rank = equal + __popcll(sames & below);
        for (int w = 0; w < kPickThreads / 64; ++w) {
            if (w < wave) rank += totals[w];
            equal += totals[w];
        }
        const bool take = i < pages && (s > prefix || (same && rank < want));
        const uint64_t takes = __ballot(take);
        __syncthreads();
        if (lane == 0) totals[wave] = __popcll(takes);
        __syncthreads();
        int to = placed + __popcll(takes & below);
        for (int w = 0; w < kPickThreads / 64; ++w) {
            if (w < wave) to += totals[w];
            placed += totals[w];
        }
        if (take) out[to] = table[i];
    }
}

template <typename T, int D>
hipError_t launch_one(const SelectProblem &p, hipStream_t stream)
{
    const int blocks = (p.width + kScorePages - 1) / kScorePages;
    hipLaunchKernelGGL((page_score_kernel<T, D>), dim3(blocks * p.B * p.kv_heads), dim3(64 * kScoreWaves), 0, stream, p);
    hipLaunchKernelGGL(page_pick_kernel, dim3(p.B * p.kv_heads), dim3(kPickThreads), 0, stream, p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(const SelectProblem &p, int head_dim, hipStream_t stream)
{
    switch (head_dim) {
    case 64: return launch_one<T, 64>(p, stream);
    case 96: return launch_one<T, 96>(p, stream);
    case 128: return launch_one<T, 128>(p, stream);
    case 256: return launch_one<T, 256>(p, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_select(const SelectProblem &p, int head_dim, marlin_dtype_t dtype, hipStream_t stream)
{
    return dtype == MARLIN_BF16 ? launch_typed<__bf16>(p, head_dim, stream) : launch_typed<_Float16>(p, head_dim, stream);
}

}  // namespace marlin
