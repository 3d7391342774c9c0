// Device parts that the append kernels share: the pieces of a head that a thread holds, their
// rotation, the slot of a position, and the page that a work-group of a prompt's
// launch takes.
#pragma once

#include "kv.h"
#include "kv_device.h"

namespace marlin {
namespace dev {

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

// The new tokens of one page of one sequence: positions lo .. hi - 1, the sequence's first new one at `start` in row `from`.
struct PageTokens {
    int b, from, start, page0, lo, hi;
};

// The mine-th page that the sequences' new tokens touch, by a work-group of NW waves; b < 0: there are fewer.  Found among the sums of
// 64 sequences' pages, then among theirs.
template <int NW>
__device__ __forceinline__ PageTokens find_page(const AppendProblem &p, int mine, int lane, int wave, int *lds_chunks)
{
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
    PageTokens x{-1, 0, 0, 0, 0, 0};
    if (chunks == 1) {
        hold(0);
    } else {
        for (int c = wave; c < chunks; c += NW) {
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
        if (chunk < 0) return x;
        hold(chunk);
    }
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + incl > mine);
    if (!past) return x;
    const int of = __builtin_ctzll(past), len = __shfl(total, of);
    x.b = chunk * 64 + of;
    x.from = __shfl(begin, of);
    x.start = len - __shfl(count, of);  // below 0 where there are more than the length says
    const int first = mine - before - (__shfl(incl, of) - __shfl(pages, of));  // of the sequence's touched pages
    x.page0 = ((x.start >> p.page_shift) + first) * (1 << p.page_shift);
    x.lo = x.page0 > x.start ? x.page0 : x.start;
    x.hi = x.page0 + (1 << p.page_shift) < len ? x.page0 + (1 << p.page_shift) : len;
    return x;
}

}  // namespace dev
}  // namespace marlin
