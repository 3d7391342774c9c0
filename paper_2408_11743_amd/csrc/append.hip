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

#include "kv.h"
#include "kv_device.h"

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

struct Pieces {
    uint32_t w[8];  // two 16-byte pieces
};

// Channels where thread `pair` of a head's D / 16 has its two pieces: where halves
// are paired, both of eight pairs; else the pieces that make neighbouring threads' accesses adjacent.
struct Where {
    int first, second;
};
__device__ __forceinline__ Where where(const AppendProblem &p, int D, int pair)
{
    if (p.interleaved) return {8 * pair, 8 * pair + D / 2};
    if (pair < p.rot / 16) return {8 * pair, 8 * pair + p.rot / 2};
    const int first = 8 * pair + p.rot / 2;  // past the rotated ones
    return {first, first + (D - p.rot) / 2};
}

template <typename T>
__device__ __forceinline__ Pieces load_pieces(const T *row, Where at)
{
    Pieces x;
    __builtin_memcpy(x.w, __builtin_assume_aligned(row + at.first, 16), 16);
    __builtin_memcpy(x.w + 4, __builtin_assume_aligned(row + at.second, 16), 16);
    return x;
}

// The same of new tokens, of which nothing is read again: non-temporal (once) where they and what becomes of them are more than the
// last-level cache holds, as what a projection has just written may still lie there, and where a piece's row of threads takes
// whole lines of 128 bytes.  Prompts of 32, 64, 128, 256 and 512 MB, 80 heads of 128 with bounds: 15.0, 34, 59, 114 and 214 us by
// ordinary loads, 19.9, 34, 57, 99 and 217 so; heads of 256: 17.9, 32.5, 63, 121 and 221, so 22, 34, 61, 102 and 219; heads of 64 lose
// at every size (256 MB: 121, 129).
template <typename T>
__device__ __forceinline__ Pieces load_new(const T *row, Where at, bool once)
{
    if (!once) return load_pieces(row, at);
    const u32x4_t a = __builtin_nontemporal_load((const u32x4_t *)(row + at.first));
    const u32x4_t b = __builtin_nontemporal_load((const u32x4_t *)(row + at.second));
    Pieces x;
    __builtin_memcpy(x.w, &a, 16);
    __builtin_memcpy(x.w + 4, &b, 16);
    return x;
}

template <typename T>
__device__ __forceinline__ void store_pieces(T *row, Where at, const Pieces &x)
{
    __builtin_memcpy(__builtin_assume_aligned(row + at.first, 16), x.w, 16);
    __builtin_memcpy(__builtin_assume_aligned(row + at.second, 16), x.w + 4, 16);
}

// Cosines and sines of the pieces' pairs: of eight (c[0], c[1]), or interleaved
// of the first piece's four and the second's.
struct Angles {
    float4_t c[2], s[2];
};
__device__ __forceinline__ Angles load_angles(const AppendProblem &p, Where at, int pos)
{
    Angles a{};
    const float *row = p.cos_sin + (int64_t)pos * p.rot;
    const int i0 = p.interleaved ? at.first / 2 : at.first, i1 = p.interleaved ? at.second / 2 : at.first + 4;
    if (at.first < p.rot) {
        a.c[0] = *(const float4_t *)(row + i0);
        a.s[0] = *(const float4_t *)(row + p.rot / 2 + i0);
    }
    if (at.second < p.rot) {
        a.c[1] = *(const float4_t *)(row + i1);
        a.s[1] = *(const float4_t *)(row + p.rot / 2 + i1);
    }
    return a;
}

template <typename T>
__device__ __forceinline__ Pieces rotate(const AppendProblem &p, const Pieces &x, const Angles &a, Where at)
{
    typedef T vec16 __attribute__((ext_vector_type(16)));
    const vec16 e = __builtin_bit_cast(vec16, x);
    vec16 y = e;
    if (p.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if ((i < 4 ? at.first : at.second) >= p.rot) continue;  // copied
            const float c = a.c[i >> 2][i & 3], s = a.s[i >> 2][i & 3], u = (float)e[2 * i], v = (float)e[2 * i + 1];
            y[2 * i] = (T)(u * c - v * s);
            y[2 * i + 1] = (T)(v * c + u * s);
        }
    } else if (at.second < p.rot) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = a.c[i >> 2][i & 3], s = a.s[i >> 2][i & 3], u = (float)e[i], v = (float)e[i + 8];
            y[i] = (T)(u * c - v * s);
            y[i + 8] = (T)(v * c + u * s);
        }
    }
    return __builtin_bit_cast(Pieces, y);
}

// A table ends at 2^30 tokens at most, and 2^24 are appended: beyond the sum of both, every new token is past the table.
__device__ __forceinline__ int clamped(int n)
{
    constexpr int kMost = (1 << 30) + (1 << 24);
    return n < 0 ? 0 : n < kMost ? n : kMost;
}

// Slot (in rows of D of the cache, kv head 0) of sequence b's position, or -1:
// the token is not appended.
__device__ __forceinline__ int64_t slot_of(const AppendProblem &p, int b, int pos)
{
    if (pos < 0 || pos >= (p.width << p.page_shift) || (p.rot > 0 && pos >= p.positions)) return -1;
    const int page = p.table[b * p.table_row + (pos >> p.page_shift)];
    if ((uint32_t)page >= (uint32_t)p.pages) return -1;
    return ((int64_t)page * p.kv_heads << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
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

    // the page: which of those that the sequences touch follows from blockIdx.x; found among the sums of 64 sequences' pages, then among theirs
    const int chunks = (p.B + 63) / 64;
    int begin = 0, count = 0, total = 0, pages = 0, incl = 0;  // of the lane's sequence: tokens, length, pages, pages up to it
    auto hold = [&](int chunk) {
        const int b = chunk * 64 + lane;
        begin = count = total = pages = 0;
        if (b < p.B) {
            begin = p.starts[b];
            int end = p.starts[b + 1];
            begin = begin < 0 ? 0 : begin < p.tokens ? begin : p.tokens;
            end = end < begin ? begin : end < p.tokens ? end : p.tokens;
            count = end - begin;
            total = clamped(p.lengths[b]);
            pages = count > 0 ? ((total - 1) >> p.page_shift) - ((total - count) >> p.page_shift) + 1 : 0;
        }
        incl = wave_scan(pages);
    };
    int chunk = 0, before = 0;
    const int q_slabs = (p.heads + kSlab - 1) / kSlab, kv_slabs = (p.kv_heads + kSlab - 1) / kSlab;
    const int in_launch = blockIdx.x / (q_slabs + 2 * kv_slabs), y = blockIdx.x - in_launch * (q_slabs + 2 * kv_slabs);
    const int mine = page_base + in_launch;
    if (chunks == 1) {
        hold(0);
    } else {
        for (int c = wave; c < chunks; c += 4) {
            hold(c);
            if (lane == 63) lds_chunks[c] = incl;
        }
        __syncthreads();
        chunk = -1;
        for (int c0 = 0; c0 < chunks && chunk < 0; c0 += 64) {
            const int c = c0 + lane < chunks ? lds_chunks[c0 + lane] : 0, i = wave_scan(c);
            const uint64_t past = __builtin_amdgcn_ballot_w64(before + i > mine);
            const int at = past ? __builtin_ctzll(past) : 63;
            if (past) chunk = c0 + at;
            before += __shfl(i, at) - (past ? __shfl(c, at) : 0);
        }
        if (chunk < 0) return;
        hold(chunk);
    }
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + incl > mine);
    if (!past) return;
    const int lane_of = __builtin_ctzll(past), b = chunk * 64 + lane_of;
    const int from = __shfl(begin, lane_of), n = __shfl(count, lane_of), len = __shfl(total, lane_of);
    const int first = mine - before - (__shfl(incl, lane_of) - __shfl(pages, lane_of));  // of the sequence's touched pages
    const int start = len - n;  // position of the first new token; below 0 where there are more than the length says
    const int page0 = ((start >> p.page_shift) + first) * (1 << p.page_shift);
    const int lo_pos = page0 > start ? page0 : start;
    const int hi_pos = page0 + (1 << p.page_shift) < len ? page0 + (1 << p.page_shift) : len;

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
