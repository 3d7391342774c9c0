// Attention of one new token per sequence over a paged key-value cache.
//
//   o_h = sum_j p_hj v_j,  p_hj = exp(scale q_h . k_j) / sum_i exp(scale q_h . k_i)
//
// One row of work is a (sequence, kv head, tile of up to 16 query heads that
// share it).  A wave takes 32 keys at a time and both products are MFMAs whose
// columns are the 16 heads, so nothing passes between lanes but the maximum:
//
//   S^T [16 keys x 16 heads] = K [16 x D] Q^T: lane (r = l % 16, g = l / 16)
//     loads 16-byte pieces of key r, and gets the scores of head r for keys
//     4g .. 4g + 3;
//   O^T [16 channels x 16 heads] += V^T [16 x 32] P^T: the contraction's order
//     is free, so lane group g contributes keys 4g .. 4g + 3 of both 16-key
//     tiles, the ones whose scores it holds; lane r loads D/16 adjacent
//     channels of them (a 16-lane row reads a whole key's row) and pairs two
//     keys' elements with v_perm, which is the whole transpose.
//
// The work is split evenly however ragged the lengths are: the rows' 32-key
// steps are numbered through and every work-group takes an equal range of
// them, found from the lengths on the device.  A work-group's eight waves split
// a row's steps and join in LDS; rows cut by range borders leave fp32 partial
// results in the workspace, and whoever arrives last joins them in order.
#include <hip/hip_runtime.h>

#include "device.h"
#include "kv.h"
#include "kv_device.h"

namespace marlin {
namespace {

using namespace dev;

// Rows shorter than twice this many steps are never cut, and no work-group
// takes less: a cut costs a round trip through the workspace, about what a
// work-group needs for as many steps.
constexpr int kMinSteps = kAttendWaves;

// Where a unit (step) of the numbering lies.
struct Place {
    int row;    // (sequence, kv head, head tile)
    int step;   // within the row
    int start;  // unit of the row's first step
};

// Steps of sequence b; a sequence without keys still has one, in which its
// outputs are written.
__device__ __forceinline__ int tokens_of(const AttendProblem &p, int b)
{
    const int n = p.lengths[b], cap = p.width << p.page_shift;
    return n < 0 ? 0 : n < cap ? n : cap;
}
__device__ __forceinline__ int steps_of(int tokens) { return tokens > 0 ? (tokens + kStepKeys - 1) / kStepKeys : 1; }

// Row and step of unit u.  Borders near a row's ends move there.
__device__ __forceinline__ Place place_of(const AttendProblem &p, int u, int lane)
{
    const int rows = p.kv_heads * p.head_tiles;  // of a sequence
    const int x = u / rows;
    int before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int c = b0 + lane < p.B ? steps_of(tokens_of(p, b0 + lane)) : 0;
        const int incl = before + wave_scan(c, lane);
        const uint64_t past = __ballot(b0 + lane < p.B && incl > x);
        if (past) {
            const int at = __builtin_ctzll(past);
            const int cb = __shfl(c, at), first = (__shfl(incl, at) - cb) * rows;
            const int r = (u - first) / cb, step = u - first - r * cb;
            const int row = (b0 + at) * rows + r, start = u - step;
            if (step < kMinSteps) return {row, 0, start};
            if (cb - step < kMinSteps) return {row + 1, 0, start + cb};
            return {row, step, start};
        }
        before = __shfl(incl, 63);
    }
    return {p.B * rows, 0, u};
}

// Smallest w with range start w * q + min(w, r) >= x.
__device__ __forceinline__ int first_at(int x, int q, int r)
{
    return x <= r * (q + 1) ? (x + q) / (q + 1) : r + (x - r * (q + 1) + q - 1) / q;
}
// Largest w with range start <= x.
__device__ __forceinline__ int last_at(int x, int q, int r)
{
    return x <= r * (q + 1) ? x / (q + 1) : r + (x - r * (q + 1)) / q;
}

template <typename T, int D, int NW>
__global__ void __launch_bounds__(64 * NW) paged_attention_kernel(const AttendProblem p)
{
    typedef Elem<T> E;
    typedef typename E::vec8 vec8;
    constexpr int kQ = D / 32;                 // 16-byte pieces of a row per lane, keys
    constexpr int kHalves = D > 128 ? 2 : 1;   // 16-byte pieces of a row per lane, values
    constexpr int kCh = D / 16 / kHalves;      // channels in each
    constexpr int kDw = kCh / 2;
    constexpr int kPad = D + 4;                // LDS row: 16 heads' float4 reach all banks
    constexpr int kItems = (kHeadTile * D / 4 + 64 * NW - 1) / (64 * NW);

    __shared__ float lds_o[NW][kHeadTile][kPad];
    __shared__ float lds_m[NW][kHeadTile], lds_l[NW][kHeadTile];
    __shared__ int lds_flag;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;

    // this work-group's range of steps
    const int rows = p.kv_heads * p.head_tiles;
    int units = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) units += b0 + lane < p.B ? steps_of(tokens_of(p, b0 + lane)) : 0;
    units = __builtin_amdgcn_readfirstlane(wave_sum(units)) * rows;
    int wgs = units / kMinSteps;
    wgs = wgs < 1 ? 1 : wgs < (int)gridDim.x ? wgs : (int)gridDim.x;
    const int wg = blockIdx.x;
    if (wg >= wgs) return;
    const int per = units / wgs, extra = units % wgs;
    auto start_of = [&](int w) { return w * per + (w < extra ? w : extra); };
    Place from = place_of(p, start_of(wg), lane), to = place_of(p, start_of(wg + 1), lane);
    from.row = __builtin_amdgcn_readfirstlane(from.row);
    from.step = __builtin_amdgcn_readfirstlane(from.step);
    from.start = __builtin_amdgcn_readfirstlane(from.start);
    to.row = __builtin_amdgcn_readfirstlane(to.row);
    to.step = __builtin_amdgcn_readfirstlane(to.step);
    to.start = __builtin_amdgcn_readfirstlane(to.start);

    const int slot_floats = kHeadTile * D + 2 * kHeadTile;
    const int last_row = to.step > 0 ? to.row : to.row - 1;
    for (int row = from.row; row <= last_row; ++row) {
        const int b = row / rows, in_b = row - b * rows;
        const int kvh = in_b / p.head_tiles, ht = in_b - kvh * p.head_tiles;
        const int heads = p.group - ht * kHeadTile < kHeadTile ? p.group - ht * kHeadTile : kHeadTile;
        const int head0 = kvh * p.group + ht * kHeadTile;
        const int tokens = tokens_of(p, b), steps = steps_of(tokens);
        const int begin = row == from.row ? from.step : 0, end = row == to.row ? to.step : steps;

        // the heads' queries: head r's channels 32t + 8g .. + 7
        vec8 qf[kQ];
        const T *q = (const T *)p.q + b * p.q_row + (head0 + r) * p.q_head + 8 * g;
#pragma unroll
        for (int t = 0; t < kQ; ++t) qf[t] = r < heads ? *(const vec8 *)(q + 32 * t) : vec8{};

        float4_t acc[kHalves * kCh];
#pragma unroll
        for (int j = 0; j < kHalves * kCh; ++j) acc[j] = float4_t{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;

        const int32_t *table = p.table + b * p.table_row + kvh * p.table_head;
        const int n = end - begin;
        const int s1 = begin + n * (wave + 1) / NW;
        for (int s = begin + n * wave / NW; s < s1 && s * kStepKeys < tokens; ++s) {
            // the step's two 16-key tiles: pages (one outside the cache counts as masked) and valid keys
            vec8 kf[2][kQ];
            uint32_t vr[2][4][kHalves][kDw];
            int valid[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int pos = s * kStepKeys + 16 * u;
                const int left = tokens - pos;
                const int page = left > 0 ? table[pos >> p.page_shift] : 0;
                const bool inside = (uint32_t)page < (uint32_t)p.pages;
                valid[u] = !inside || left < 0 ? 0 : left < 16 ? left : 16;
                const int64_t at = (((int64_t)(inside ? page : 0) * p.kv_heads + kvh) << p.page_shift) +
                                   (pos & ((1 << p.page_shift) - 1));
                const T *k = (const T *)p.k + at * D, *v = (const T *)p.v + at * D;
#pragma unroll
                for (int t = 0; t < kQ; ++t) kf[u][t] = *(const vec8 *)(k + (r * D + 8 * g) + 32 * t);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf)
                        load_dwords<kDw>(vr[u][i][hf], v + (4 * g * D + kCh * r) + i * D + 128 * hf);
            }
            float4_t sc[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                sc[u] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < kQ; ++t) sc[u] = E::mfma(kf[u][t], qf[t], sc[u]);
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[u][i] *= p.scale_log2;
            }
            if (valid[0] < 16 || valid[1] < 16) {
                // whatever a masked slot holds (an infinity, not a number) stays out of both products
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (4 * g + i >= valid[u]) {
                            sc[u][i] = -INFINITY;
#pragma unroll
                            for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                                for (int w = 0; w < kDw; ++w) vr[u][i][hf][w] = 0;
                        }
            }
            float top = m;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[u][i]);
            top = max_over_groups(top);
            const float ref = top == -INFINITY ? 0.f : top;  // nothing but -inf so far: weights 0
            const float keep = __builtin_amdgcn_exp2f(m - ref);
            m = top;
            float pr[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) pr[u][i] = __builtin_amdgcn_exp2f(sc[u][i] - ref);
            l = l * keep + ((pr[0][0] + pr[0][1]) + (pr[0][2] + pr[0][3])) + ((pr[1][0] + pr[1][1]) + (pr[1][2] + pr[1][3]));
            vec8 pf;
#pragma unroll
            for (int e = 0; e < 8; ++e) pf[e] = (T)pr[e >> 2][e & 3];
#pragma unroll
            for (int j = 0; j < kHalves * kCh; ++j) acc[j] *= keep;
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                for (int j = 0; j < kCh; ++j) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w[e] = __builtin_amdgcn_perm(vr[e >> 1][2 * (e & 1) + 1][hf][j >> 1], vr[e >> 1][2 * (e & 1)][hf][j >> 1],
                                                     (j & 1) ? 0x07060302u : 0x05040100u);
                    acc[hf * kCh + j] = E::mfma(__builtin_bit_cast(vec8, u32x4_t{w[0], w[1], w[2], w[3]}), pf, acc[hf * kCh + j]);
                }
        }
        l = sum_over_groups(l);

        // the waves' results: lane (r, g) holds head r's channels kCh (4g + i) + j
#pragma unroll
        for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < kCh; ++j) lds_o[wave][r][128 * hf + kCh * (4 * g + i) + j] = acc[hf * kCh + j][i];
        if (g == 0) {
            lds_m[wave][r] = m;
            lds_l[wave][r] = l;
        }
        __syncthreads();
        const bool whole = begin == 0 && end == steps;
        // contributors of a row that is cut: those whose ranges start within it, and the one before
        int w_first = 0, others = 0;
        if (!whole) {
            const int start = row == from.row ? from.start : to.start;
            w_first = first_at(start + kMinSteps, per, extra) - 1;
            others = last_at(start + steps - kMinSteps, per, extra) - w_first;
        }
        float *const slot = p.partials + ((int64_t)wg * 2 + (begin > 0 ? 0 : 1)) * slot_floats;
        float4_t res[kItems];
        float top[kItems], sum[kItems];
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const int it = tid + k * 64 * NW, h = it / (D / 4), d = it % (D / 4) * 4;
            if (h >= heads) continue;
            float t = -INFINITY, s = 0.f;
            float4_t o{0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < NW; ++w) t = fmaxf(t, lds_m[w][h]);
            const float ref = t == -INFINITY ? 0.f : t;
            for (int w = 0; w < NW; ++w) {
                const float f = __builtin_amdgcn_exp2f(lds_m[w][h] - ref);
                s += f * lds_l[w][h];
                o += f * *(const float4_t *)&lds_o[w][h][d];
            }
            res[k] = o;
            top[k] = t;
            sum[k] = s;
            if (!whole) {
                store_partial16(slot, wave + k * NW, lane, o);
                if (d == 0) {
                    store_float(slot + kHeadTile * D + h, t);
                    store_float(slot + kHeadTile * D + kHeadTile + h, s);
                }
            }
        }
        if (!whole) {
            wait_vmcnt<0>();
            __syncthreads();
            if (tid == 0) {
                uint32_t *const ctr = p.counters + kCounterStride * w_first;
                const bool last = __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)others;
                if (last) __hip_atomic_store(ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                lds_flag = last;
            }
            __syncthreads();
            if (lds_flag) {
                // in the order of the ranges, so the same inputs give the same bits
#pragma unroll
                for (int k = 0; k < kItems; ++k) {
                    const int it = tid + k * 64 * NW, h = it / (D / 4);
                    if (h >= heads) continue;
                    float t = -INFINITY, s = 0.f;
                    float4_t o{0.f, 0.f, 0.f, 0.f};
                    for (int w = w_first; w <= w_first + others; ++w) {
                        const float *from_w = p.partials + ((int64_t)w * 2 + (w == w_first ? 1 : 0)) * slot_floats;
                        const float mw = load_float(from_w + kHeadTile * D + h), lw = load_float(from_w + kHeadTile * D + kHeadTile + h);
                        const float4_t ow = load_partial16(from_w, wave + k * NW, lane);
                        const float nt = fmaxf(t, mw), ref = nt == -INFINITY ? 0.f : nt;
                        const float fo = __builtin_amdgcn_exp2f(t - ref), fw = __builtin_amdgcn_exp2f(mw - ref);
                        s = s * fo + lw * fw;
                        o = o * fo + ow * fw;
                        t = nt;
                    }
                    res[k] = o;
                    top[k] = t;
                    sum[k] = s;
                }
            }
        }
        if (whole || lds_flag) {
#pragma unroll
            for (int k = 0; k < kItems; ++k) {
                const int it = tid + k * 64 * NW, h = it / (D / 4), d = it % (D / 4) * 4;
                if (h >= heads) continue;
                const int64_t at = (int64_t)b * p.heads + head0 + h;
                const float inv = sum[k] == 0.f ? 0.f : 1.f / sum[k];  // no key: zero
                typedef T vec4 __attribute__((ext_vector_type(4)));
                vec4 y;
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = (T)(res[k][i] * inv);
                *(vec4 *)((T *)p.out + at * D + d) = y;
                if (p.lse && d == 0) p.lse[at] = (top[k] + __builtin_amdgcn_logf(sum[k])) * 0.693147180559945f;
            }
        }
        __syncthreads();  // before the next row's results go to LDS
    }
}

template <typename T, int D>
hipError_t launch_one(const AttendProblem &p, int cus, hipStream_t stream)
{
    const int grid = (cus < kKvMaxCus ? cus : kKvMaxCus) * kAttendGroupsPerCu;
    hipLaunchKernelGGL((paged_attention_kernel<T, D, kAttendWaves>), dim3(grid), dim3(64 * kAttendWaves), 0, stream, p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(const AttendProblem &p, int head_dim, int cus, hipStream_t stream)
{
    switch (head_dim) {
    case 64: return launch_one<T, 64>(p, cus, stream);
    case 96: return launch_one<T, 96>(p, cus, stream);
    case 128: return launch_one<T, 128>(p, cus, stream);
    case 256: return launch_one<T, 256>(p, cus, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_attend(const AttendProblem &p, int head_dim, marlin_dtype_t dtype, int cus, hipStream_t stream)
{
    return dtype == MARLIN_BF16 ? launch_typed<__bf16>(p, head_dim, cus, stream)
                                : launch_typed<_Float16>(p, head_dim, cus, stream);
}

}  // namespace marlin
