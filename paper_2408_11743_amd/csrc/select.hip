// The pages a new token attends to: each page is scored by the largest product
// that the bounds of its keys (smallest and largest per channel) allow with a
// query of the kv head's group,
//
//   score = max_h sum_c (q_hc > 0 ? q_hc hi_c : q_hc lo_c)
//         = max_h (min(q_h, 0) . lo + max(q_h, 0) . hi)   where the bounds are finite,
//
// a product over 2 D channels for the MFMAs, and the best `select` are kept in the
// order of their positions.
//
// Latency bounds both kernels: 8 rows of 4063 pages are scored in 6.2 us (16.6
// MB) and picked from in 6.4, 256 rows of 10 .. 1875 in 14.6 (48.7 MB) and 6.1.
#include <hip/hip_runtime.h>

#include "kv.h"
#include "kv_device.h"

namespace marlin {
namespace {

using namespace dev;

// Waves are independent: small work-groups come and go faster (32 sequences of up to 60000 tokens selected and attended
// in 62.7 us with two, 64.1 four, 65.9 eight).
constexpr int kScoreWaves = 2;

__device__ __forceinline__ int pages_of(const SelectProblem &p, int b)
{
    const int n = p.lengths[b], cap = p.width << p.page_shift;
    const int len = n < 0 ? 0 : n < cap ? n : cap;
    return (len + (1 << p.page_shift) - 1) >> p.page_shift;
}

// fp32 to integers in the same order, from 1 to 2^32 - 3; a score that is not a
// number is 2^32 - 2, no page 0.
constexpr uint32_t kNoPage = 0u, kNan = 0xFFFFFFFEu;
__device__ __forceinline__ uint32_t score_key(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);  // -0 and 0 are equal
    return x != x ? kNan : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// A wave scores 16 pages: lane (r = l % 16, g = l / 16) loads 16-byte pieces of
// page r's bounds and gets the products of heads 4g .. 4g + 3 with it.  (Two,
// four or eight tiles a wave, the queries loaded once: 32 sequences of up to 60000 tokens
// selected and attended in 69.0, 77.8, 86.1 us when one took 68.8.)
template <typename T, int D>
__global__ void __launch_bounds__(64 * kScoreWaves) page_score_kernel(const SelectProblem p, int blocks)
{
    typedef typename Elem<T>::vec8 vec8;
    constexpr int kQ = D / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int row = blockIdx.x / blocks, b = row / p.kv_heads, kvh = row - b * p.kv_heads;
    const int page0 = ((int)(blockIdx.x - row * blocks) * kScoreWaves + wave) * 16, at = page0 + r;
    // The length first: most of a ragged batch's work-groups lie past it (32 sequences of 300 .. 60000 tokens in pages of 32
    // selected in 17.3 us, with entries and queries under way while the length is in 21.4; one of 32000 in 9.2 both ways).
    const int pages = pages_of(p, b);
    if (pages <= p.select || page0 >= pages) return;
    const int page = at < pages ? p.table[b * p.table_row + at] : -1;
    const T *q0 = (const T *)p.q + b * p.q_row + (kvh * p.group + r) * p.q_head + 8 * g;
    vec8 qf[kQ];
#pragma unroll
    for (int t = 0; t < kQ; ++t) qf[t] = r < p.group ? *(const vec8 *)(q0 + 32 * t) : vec8{};
    const bool inside = (uint32_t)page < (uint32_t)p.pages;
    const T *box = (const T *)p.bounds + ((int64_t)(inside ? page : 0) * p.kv_heads + kvh) * 2 * D + 8 * g;
    vec8 lo[kQ], hi[kQ];
#pragma unroll
    for (int t = 0; t < kQ; ++t) {
        lo[t] = *(const vec8 *)(box + 32 * t);
        hi[t] = *(const vec8 *)(box + D + 32 * t);
    }
    float best = -INFINITY;
    bool odd = false;
    for (int h0 = 0; h0 < p.group; h0 += 16) {
        if (h0 > 0)
#pragma unroll
            for (int t = 0; t < kQ; ++t)
                qf[t] = h0 + r < p.group ? *(const vec8 *)(q0 + h0 * p.q_head + 32 * t) : vec8{};
        float4_t s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < kQ; ++t) {
            const vec8 x = qf[t];
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
                odd |= !(fabsf(s[i]) < INFINITY);
            }
    }
    auto of_page = [&](bool x) -> bool {  // in any of the page's four lanes
        const uint64_t in = __builtin_amdgcn_ballot_w64(x);
        return (in >> r | in >> (r + 16) | in >> (r + 32) | in >> (r + 48)) & 1;
    };
    best = max_over_groups(best);
    // The products also take what the formula leaves out, times zero: of a bound that is infinite or no number they are no number or
    // infinite.  Such a page, a rare one, is scored anew as the formula says.
    odd = of_page(odd) && inside;
    bool nan = false;
    if (__any(odd)) {
        float anew = -INFINITY;
#pragma unroll 1
        for (int h = 0; h < p.group; ++h) {
            const T *q = (const T *)p.q + b * p.q_row + (kvh * p.group + h) * p.q_head + 8 * g;
            float sum = 0.f;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                const vec8 x = *(const vec8 *)(q + c), least = *(const vec8 *)(box + c), most = *(const vec8 *)(box + D + c);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += (float)x[e] * (x[e] > (T)0.f ? (float)most[e] : (float)least[e]);
            }
            sum = sum_over_groups(sum);
            anew = fmaxf(anew, sum);
            nan |= sum != sum;
        }
        if (odd) best = anew;
        nan &= odd;
    }
    if (g == 0 && at < pages) p.scores[(int64_t)row * p.width + at] = !inside ? kNoPage : nan ? kNan : score_key(best);
}

constexpr int kPickThreads = 512, kPickWaves = kPickThreads / 64;

struct Counts {
    int a, b;
};
// Sums over the work-group's lanes before this one.
__device__ __forceinline__ Counts group_scan(Counts x, Counts *waves)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Counts i{wave_scan(x.a), wave_scan(x.b)};
    if (lane == 63) waves[wave] = i;
    __syncthreads();
    Counts before{i.a - x.a, i.b - x.b};
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) {
        before.a += w < wave ? waves[w].a : 0;
        before.b += w < wave ? waves[w].b : 0;
    }
    return before;
}

// The wave's smallest (largest) value, in lane 63.
template <bool MIN>
__device__ __forceinline__ uint32_t wave_end(uint32_t x)
{
    auto with = [&](uint32_t y) { x = MIN ? (y < x ? y : x) : (y > x ? y : x); };
    with((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x111, 0xf, 0xf, false));
    with((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x112, 0xf, 0xf, false));
    with((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x114, 0xf, 0xf, false));
    with((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x118, 0xf, 0xf, false));
    with((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x142, 0xa, 0xf, false));
    with((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x143, 0xc, 0xf, false));
    return x;
}

// One work-group per (sequence, kv head) finds the score that the select - 1 best
// pages but the last reach: counts of the scores in 2048 equal parts
// of their range, then of the part that holds it, until the part is one score or wanted whole
// (the parts follow the range, so that few scores meet in one counter); then every page above it and the first ones equal to
// it, in order.  A thread's pages are adjacent; HELD of them, it reads their scores and entries
// while the length is under way, in vectors, and keeps them in registers.  Of more (HELD 0), scores are read in each
// pass, and the entries of the chosen in the end (8125 pages so: 37.6 us with scores and attention, HELD 26.3).
constexpr int kPickBins = 2048;

// N adjacent words, in vectors aligned to a word.
template <int N, typename T>
__device__ __forceinline__ void load_unaligned(T (&to)[N], const T *from)
{
    constexpr int kVec = N < 4 ? N : 4;
    typedef T vec __attribute__((ext_vector_type(kVec), aligned(4)));
#pragma unroll
    for (int i = 0; i < N; i += kVec) {
        const vec x = *(const vec *)(from + i);
#pragma unroll
        for (int k = 0; k < kVec; ++k) to[i + k] = x[k];
    }
}

template <int HELD>
__global__ void __launch_bounds__(kPickThreads) page_pick_kernel(const SelectProblem p, int row_base)
{
    __shared__ int bins[kPickBins], found[3];
    __shared__ Counts waves[2][kPickWaves];
    __shared__ uint32_t ends[2][kPickWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = row_base + blockIdx.x, b = row / p.kv_heads, kvh = row % p.kv_heads;
    const int32_t *table = p.table + b * p.table_row;
    const uint32_t *scores = p.scores + (int64_t)row * p.width;
    uint32_t held[HELD ? HELD : 1];
    int32_t entry[HELD ? HELD : 1];
    if constexpr (HELD > 0) {
        const int first = HELD * tid;
        if (first + HELD <= p.width) {
            load_unaligned(held, scores + first);
            load_unaligned(entry, table + first);
        } else {
#pragma unroll
            for (int k = 0; k < HELD; ++k)
                if (first + k < p.width) {
                    held[k] = scores[first + k];
                    entry[k] = table[first + k];
                }
        }
    }
    const int pages = pages_of(p, b);
    int32_t *out = p.chosen + (int64_t)row * p.select;
    if (kvh == 0 && tid == 0) {
        const int n = p.lengths[b], cap = p.width << p.page_shift, len = n < 0 ? 0 : n < cap ? n : cap;
        p.chosen_lengths[b] = pages > p.select ? len - ((pages - p.select) << p.page_shift) : len;
    }
    if (pages <= p.select) {
        for (int i = tid; i < p.select; i += kPickThreads) out[i] = i < pages ? table[i] : -1;
        return;
    }
    const int n = pages - 1;  // the last page is chosen anyway
    const int per = HELD ? HELD : (n + kPickThreads - 1) / kPickThreads, i0 = tid * per < n ? tid * per : n, i1 = i0 + per < n ? i0 + per : n;
    // the scores, a thread's in order (any: in whatever order)
    auto each = [&](bool any, auto &&f) {
        if constexpr (HELD > 0) {
#pragma unroll
            for (int k = 0; k < HELD; ++k)
                if (i0 + k < i1) f(k, held[k]);
        } else if (any) {
#pragma unroll 8
            for (int i = tid; i < n; i += kPickThreads) f(i, scores[i]);
        } else {
#pragma unroll 4
            for (int i = i0; i < i1; ++i) f(i, scores[i]);
        }
    };
    int want = p.select - 1;  // of the pages with scores from lo to hi; those above hi are chosen
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    auto widen = [&](uint32_t s) {
        lo = s < lo ? s : lo;
        hi = s > hi ? s : hi;
    };
    each(true, [&](int, uint32_t s) { widen(s); });
    for (int i = tid; i < kPickBins; i += kPickThreads) bins[i] = 0;
    lo = wave_end<true>(lo);
    hi = wave_end<false>(hi);
    if (lane == 63) {
        ends[0][wave] = lo;
        ends[1][wave] = hi;
    }
    __syncthreads();
    lo = ends[0][0];
    hi = ends[1][0];
#pragma unroll
    for (int w = 1; w < kPickWaves; ++w) {
        lo = ends[0][w] < lo ? ends[0][w] : lo;
        hi = ends[1][w] > hi ? ends[1][w] : hi;
    }
    uint32_t bar = 0xFFFFFFFFu;  // chosen: scores above it, and the first `want` equal to it
    while (want > 0) {
        const int bits = 32 - __clz(hi - lo | 1u), shift = bits > 11 ? bits - 11 : 0;
        each(true, [&](int, uint32_t s) {
            if (s >= lo && s <= hi) atomicAdd(&bins[(s - lo) >> shift], 1);
        });
        __syncthreads();
        // thread t: bins 4 (511 - t) .. + 3, from the top
        constexpr int kPer = kPickBins / kPickThreads;
        int c[kPer], sum = 0;
#pragma unroll
        for (int k = 0; k < kPer; ++k) sum += c[k] = bins[kPickBins - 1 - kPer * tid - k];
        int upto = group_scan({sum, 0}, waves[0]).a;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int bin = kPickBins - 1 - kPer * tid - k;
            bins[bin] = 0;
            if (upto < want && want <= upto + c[k]) {
                found[0] = bin;
                found[1] = upto;
                found[2] = c[k];
            }
            upto += c[k];
        }
        __syncthreads();
        const uint32_t first = lo + ((uint32_t)found[0] << shift);
        want -= found[1];
        const bool whole = want == found[2];
        if (shift == 0 || whole) {
            bar = first;
            if (whole) want = n;  // all from `first` on
            break;
        }
        lo = first;
        hi = hi - first < 1u << shift ? hi : first + ((1u << shift) - 1);
        __syncthreads();
    }
    if (bar != 0xFFFFFFFFu) {
        Counts mine{0, 0};
        each(false, [&](int, uint32_t s) {
            mine.a += s > bar;
            mine.b += s == bar;
        });
        const Counts before = group_scan(mine, waves[1]);
        int e = before.b, to = before.a + (e < want ? e : want);
        const bool listed = !HELD && p.select <= kPickBins;  // then the table is read for all of them together
        each(false, [&](int i, uint32_t s) {
            if (s > bar || (s == bar && e < want)) {
                if (HELD)
                    out[to] = entry[i];
                else if (listed)
                    bins[to] = i;
                else
                    out[to] = table[i];
                ++to;
            }
            e += s == bar;
        });
        if (listed) {
            __syncthreads();
            for (int k = tid; k < p.select - 1; k += kPickThreads) out[k] = table[bins[k]];
        }
    }
    if (tid == 0) out[p.select - 1] = table[pages - 1];
}

template <typename T, int D>
hipError_t launch_one(const SelectProblem &p, hipStream_t stream)
{
    constexpr int kPer = 16 * kScoreWaves;
    const int blocks = (p.width + kPer - 1) / kPer;
    // no scores where every sequence keeps all the pages it can have (one sequence of 21 tokens: 9.0 us with the
    // attention, 11.3 with a launch that finds nothing to do)
    SelectProblem q = p;
    if (p.width > p.select) {
        int n = blocks;
        void *args[] = {&q, &n};
        const hipError_t e = hipLaunchKernel((const void *)&page_score_kernel<T, D>, dim3(blocks * p.B * p.kv_heads),
                                             dim3(64 * kScoreWaves), args, 0, stream);
        if (e != hipSuccess) return e;
    }
    // entries and scores that a thread of the pick holds
    const void *const pick = p.width <= kPickThreads        ? (const void *)&page_pick_kernel<1>
                             : p.width <= 2 * kPickThreads  ? (const void *)&page_pick_kernel<2>
                             : p.width <= 4 * kPickThreads  ? (const void *)&page_pick_kernel<4>
                             : p.width <= 8 * kPickThreads  ? (const void *)&page_pick_kernel<8>
                             : p.width <= 16 * kPickThreads ? (const void *)&page_pick_kernel<16>
                             : p.width <= 32 * kPickThreads ? (const void *)&page_pick_kernel<32>
                                                            : (const void *)&page_pick_kernel<0>;
    constexpr int kMost = 1 << 22;  // rows of a launch, which takes less than 2^32 threads
    const int rows = p.B * p.kv_heads;
    for (int base = 0; base < rows; base += kMost) {
        void *args[] = {&q, &base};
        const hipError_t e = hipLaunchKernel(pick, dim3(rows - base < kMost ? rows - base : kMost), dim3(kPickThreads), args, 0, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
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
