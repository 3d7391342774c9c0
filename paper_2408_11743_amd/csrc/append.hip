// New tokens into the paged key-value cache: queries and keys rotated by their
// positions, (x, y) -> (x cos a - y sin a, y cos a + x sin a) in fp32 with one
// rounding, keys and values written to their pages, and the pages' bounds (the
// smallest and largest key per channel) widened.
//
// A head is D / 16 threads, each with two 16-byte pieces that hold eight pairs.
// Nothing is read twice but the angles.  Prompts are bound by memory (24
// prompts of up to 4096 tokens, 64 + 16 heads of 128 with bounds, 605 MB read and written:
// 124 us, 4.9 TB/s, and 111 where the queries' last-level lines are written again; a large copy
// reaches 4.8), a token per sequence by launch latency (32 + 16 heads: 2.4 us; 128
// sequences of 64 + 16 heads with bounds: 4.0).
#include <hip/hip_runtime.h>

#include "append.h"
#include "kv.h"

namespace marlin {
namespace {

using namespace dev;

typedef int16_t short2_t __attribute__((ext_vector_type(2)));

// 16-bit floats, two to a dword, to integers in the same order (and back): the
// magnitude bits of negative ones are inverted.
__device__ __forceinline__ uint32_t ordered(uint32_t x) { return x ^ ((x >> 15) & 0x00010001u) * 0x7FFFu; }

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(short2_t, a), __builtin_bit_cast(short2_t, b)));
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(short2_t, a), __builtin_bit_cast(short2_t, b)));
}

// ---- one token per sequence ----
template <typename T, int D>
__global__ void __launch_bounds__(256) append_token_kernel(const AppendProblem p)
{
    constexpr int kPairs = D / 16, kHeads = 256 / kPairs;
    const int pair = threadIdx.x % kPairs, slabs = (p.heads + 2 * p.kv_heads + kHeads - 1) / kHeads;
    const int b = blockIdx.x / slabs, h = blockIdx.x % slabs * kHeads + threadIdx.x / kPairs;
    if (threadIdx.x >= kHeads * kPairs || h >= p.heads + 2 * p.kv_heads) return;
    const int pos = clamped(p.lengths[b]) - 1;
    const int64_t slot = slot_of(p, b, pos);
    const Where at = where(p, D, pair);
    if (h < p.heads) {
        Pieces x{};
        if (slot >= 0)
            x = rotate<T>(p, load_pieces((const T *)p.q + b * p.q_row + h * p.q_head, at), load_angles(p, at, pos), at);
        store_pieces((T *)p.q_out + ((int64_t)b * p.heads + h) * D, at, x);
        return;
    }
    if (slot < 0) return;
    const int kh = h - p.heads < p.kv_heads ? h - p.heads : h - p.heads - p.kv_heads;
    const int64_t to = (slot + ((int64_t)kh << p.page_shift)) * D;
    if (h >= p.heads + p.kv_heads) {
        store_pieces((T *)p.v_cache + to, at, load_pieces((const T *)p.v + b * p.v_row + kh * p.v_head, at));
        return;
    }
    Pieces x = rotate<T>(p, load_pieces((const T *)p.k + b * p.k_row + kh * p.k_head, at), load_angles(p, at, pos), at);
    store_pieces((T *)p.k_cache + to, at, x);
    if (p.bounds) {
        T *lo = (T *)p.bounds + ((slot >> p.page_shift) + kh) * 2 * D, *hi = lo + D;
        Pieces y = x;
        if (slot & ((1 << p.page_shift) - 1)) {
            const Pieces old_lo = load_pieces(lo, at), old_hi = load_pieces(hi, at);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t o = ordered(x.w[i]);
                x.w[i] = ordered(min2(ordered(old_lo.w[i]), o));
                y.w[i] = ordered(max2(ordered(old_hi.w[i]), o));
            }
        }
        store_pieces(lo, at, x);
        store_pieces(hi, at, y);
    }
}

// ---- any number of tokens per sequence ----
// A work-group takes the new tokens of one page of one sequence and four heads
// of q, of k or of v: each wave some tokens, whose four heads it reads before
// it writes any.  Keys with bounds are a head a wave instead, so that a page's
// bounds are one wave's: kept in its registers and joined across its lanes (all
// four heads' in every wave, joined in LDS: 64 registers, which spilled, 130 us where the
// prompts above take 111).  Neighbouring work-groups take the heads of one page, which lie side by side in
// the tokens' rows (neighbouring pages instead: 9 % more).
// Slabs of two heads: 24 % more, of eight 5 % more.
constexpr int kSlab = 4;

template <typename T, int D>
__global__ void __launch_bounds__(256, 4) append_prompt_kernel(const AppendProblem p, bool once, int page_base)
{
    constexpr int kPairs = D / 16;
    constexpr int kTokens = D == 64 ? 16 : D == 256 ? 4 : 8;  // of a wave at a time
    __shared__ int lds_chunks[kKvMaxBatch / 64];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int pair = lane % kPairs, slot = lane / kPairs;

    const int q_slabs = (p.heads + kSlab - 1) / kSlab, kv_slabs = (p.kv_heads + kSlab - 1) / kSlab;
    const int in_launch = blockIdx.x / (q_slabs + 2 * kv_slabs), y = blockIdx.x - in_launch * (q_slabs + 2 * kv_slabs);
    const PageTokens part = find_page<4>(p, page_base + in_launch, lane, wave, lds_chunks);
    if (part.b < 0) return;
    const int b = part.b, from = part.from, start = part.start, page0 = part.page0, lo_pos = part.lo, hi_pos = part.hi;

    const int kind = y < q_slabs ? 0 : y < q_slabs + kv_slabs ? 1 : 2;
    const int h0 = (kind == 0 ? y : kind == 1 ? y - q_slabs : y - q_slabs - kv_slabs) * kSlab;
    const int nh = (kind == 0 ? p.heads : p.kv_heads) - h0 < kSlab ? (kind == 0 ? p.heads : p.kv_heads) - h0 : kSlab;
    const T *src = (const T *)(kind == 0 ? p.q : kind == 1 ? p.k : p.v);
    const int64_t row = kind == 0 ? p.q_row : kind == 1 ? p.k_row : p.v_row;
    const int64_t head = kind == 0 ? p.q_head : kind == 1 ? p.k_head : p.v_head;
    const Where at = where(p, D, pair);

    if (!(kind == 1 && p.bounds)) {
        if (slot >= kTokens) return;
        for (int pos = lo_pos + wave * kTokens + slot; pos < hi_pos; pos += 4 * kTokens) {
            const int64_t t = from + (pos - start);
            const int64_t to = slot_of(p, b, pos);
            if (to < 0) {
                if (kind == 0)
                    for (int j = 0; j < nh; ++j) store_pieces((T *)p.q_out + (t * p.heads + h0 + j) * D, at, Pieces{});
                continue;
            }
            Pieces x[kSlab];
#pragma unroll
            for (int j = 0; j < kSlab; ++j)
                if (j < nh) x[j] = load_new(src + t * row + (h0 + j) * head, at, once);
            if (kind == 0) {
                const Angles a = load_angles(p, at, pos);
#pragma unroll
                for (int j = 0; j < kSlab; ++j)
                    if (j < nh) store_pieces((T *)p.q_out + (t * p.heads + h0 + j) * D, at, rotate<T>(p, x[j], a, at));
                continue;
            }
            if (kind == 1) {
                const Angles a = load_angles(p, at, pos);
#pragma unroll
                for (int j = 0; j < kSlab; ++j) x[j] = rotate<T>(p, x[j], a, at);
            }
            T *cache = (T *)(kind == 1 ? p.k_cache : p.v_cache) + to * D;
#pragma unroll
            for (int j = 0; j < kSlab; ++j)
                if (j < nh) store_pieces(cache + ((int64_t)(h0 + j) << p.page_shift) * D, at, x[j]);
        }
        return;
    }

    // keys with bounds: a head is one wave's
    if (wave >= nh) return;
    const int h = h0 + wave;
    uint32_t lo[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo[i] = 0x7FFF7FFFu;
        hi[i] = 0x80008000u;
    }
    bool kept = false;
    if (slot < kTokens) {
        for (int pos = lo_pos + slot; pos < hi_pos; pos += kTokens) {
            const int64_t to = slot_of(p, b, pos);
            if (to < 0) continue;
            const Pieces x = load_new(src + (int64_t)(from + (pos - start)) * row + h * head, at, once);
            const Pieces y = rotate<T>(p, x, load_angles(p, at, pos), at);
            store_pieces((T *)p.k_cache + (to + ((int64_t)h << p.page_shift)) * D, at, y);
            kept = true;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t o = ordered(y.w[i]);
                lo[i] = min2(lo[i], o);
                hi[i] = max2(hi[i], o);
            }
        }
    }
    if (!__any(kept)) return;
#pragma unroll
    for (int d = kTokens / 2; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            lo[i] = min2(lo[i], __shfl(lo[i], (lane + kPairs * d) & 63));
            hi[i] = max2(hi[i], __shfl(hi[i], (lane + kPairs * d) & 63));
        }
    if (slot > 0) return;
    const int page = p.table[b * p.table_row + (page0 >> p.page_shift)];
    T *to_lo = (T *)p.bounds + ((int64_t)page * p.kv_heads + h) * 2 * D, *to_hi = to_lo + D;
    Pieces x, z;
    if (lo_pos > page0) {
        const Pieces old_lo = load_pieces(to_lo, at), old_hi = load_pieces(to_hi, at);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            lo[i] = min2(lo[i], ordered(old_lo.w[i]));
            hi[i] = max2(hi[i], ordered(old_hi.w[i]));
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x.w[i] = ordered(lo[i]);
        z.w[i] = ordered(hi[i]);
    }
    store_pieces(to_lo, at, x);
    store_pieces(to_hi, at, z);
}

template <typename T, int D>
hipError_t launch_one(const AppendProblem &p, hipStream_t stream)
{
    AppendProblem q = p;
    if (!p.starts) {
        constexpr int kHeads = 256 / (D / 16);
        const int slabs = (p.heads + 2 * p.kv_heads + kHeads - 1) / kHeads;
        void *args[] = {&q};
        return hipLaunchKernel((const void *)&append_token_kernel<T, D>, dim3((uint32_t)p.B * slabs), dim3(256), args, 0, stream);
    }
    // a sequence of n tokens touches at most n / page size + 2 pages
    const int pages = (p.tokens >> p.page_shift) + 2 * (p.B < p.tokens ? p.B : p.tokens);
    const int slabs = (p.heads + kSlab - 1) / kSlab + 2 * ((p.kv_heads + kSlab - 1) / kSlab);
    bool once = D % 128 == 0 && (int64_t)p.tokens * (p.heads + 2 * p.kv_heads) * D * 2 > ((int64_t)128 << 20);
    const int most = (1 << 24) / slabs - 1;  // pages of a launch, which takes less than 2^32 threads
    for (int base = 0; base < pages; base += most) {
        void *args[] = {&q, &once, &base};
        const uint32_t n = pages - base < most ? pages - base : most;
        const hipError_t e = hipLaunchKernel((const void *)&append_prompt_kernel<T, D>, dim3(n * slabs), dim3(256), args, 0, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t launch_typed(const AppendProblem &p, int head_dim, hipStream_t stream)
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

hipError_t launch_append(const AppendProblem &p, int head_dim, marlin_dtype_t dtype, hipStream_t stream)
{
    return dtype == MARLIN_BF16 ? launch_typed<__bf16>(p, head_dim, stream) : launch_typed<_Float16>(p, head_dim, stream);
}

}  // namespace marlin
