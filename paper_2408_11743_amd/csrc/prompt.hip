// Attention of several new tokens per sequence over a paged key-value cache: prompts,
// their chunks, drafted tokens.
//
//   o_t = sum_j p_tj v_j,  p_tj = exp(scale q_t . k_j) / sum_i exp(scale q_t . k_i),  j up to t's position, and through a window
//
// A tile of work is rows of one sequence and kv head: its tokens by the query heads that share the
// kv head (row r: token r / group, head r % group), so keys and values are read once for all of
// them.  Both products are MFMAs with the rows as columns,
//
//   S^T [keys x rows] = K Q^T,  O^T [channels x rows] += V^T P^T,
//
// so a row's scores lie in few lanes, which need no exchange but for the maximum, and a lane's
// scores are the operand of the second product as they are: the contraction's order is free, and V^T
// is laid out in the order in which the lanes hold the keys.
//
// The tiles of a call are numbered from the sequences' starts on the device; a work-group finds its tile by
// scans, the longest of a sequence first.  Where there are few tiles, their keys are split into parts of one length, a work-group
// each, which leave partial results in the workspace; a second launch joins those in order.
//
// Weights go to the second product in the cache's type.  Up to kTwoRows rows a sequence and kv head (the mean) in two parts, as those of one token
// per sequence (attend.hip: 21 bits in float16, 15 in bfloat16), so that drafted tokens are weighed as decoding weighs them: 32 sequences'
// drafts over 8 bits 39.9 us, rounded once 39.4; one of 60000 tokens 41.8 and 38.9.  Of more rows they are rounded once, an error of half a step of each weight, as
// the output's own, and averaged over the keys; float16's are times 2^11, so that they are no subnormals until 2^-25 of the maximum, and lost
// below 2^-36: 2^20 keys that are lost are less than half a step of the sum.  Second parts would take half the matrix products again: a prompt of 8192
// tokens 854 us for 644, windowed ones 126 for 101, chunks over 8 bits 836 for 640, where the errors against 64 bits (2-norm) are 2.03e-4 for 2.05e-4 and
// in bfloat16 1.65e-3 for 1.69e-3, nearly all of it the output's rounding.  Over 8 bits a weight is times its block's scale of values in all of
// this.  Scores, maxima, sums and results are fp32.
//
// Many rows are bound by power: a prompt of 8192 tokens, 32 heads over 8 of 128 channels (550 GFLOP), takes 602 to 655 us, 0.84 to 0.91 PFLOP/s, where
// a matrix product of 8192 cubed takes 1.11; with inputs of zero, a fifth less.  Per score the 32 MFMAs of 64 keys are 45 % of the SIMDs'
// cycles, the softmax's vector instructions most of the rest, beside them from the other work-group.  Two columns of rows a wave, one wave a SIMD:
// 780 us; eight waves a work-group: 2 % less, but 20 % more where tiles are few.  Four prompts, 2270 tokens, 64 heads over 8, through a window of 1024: 97 to 102 us;
// four chunks of 512 tokens behind up to 16384 in 8 bits (535 GFLOP): 605 to 650.  Few rows are bound by memory and the latency of two launches: 32 sequences of up to
// 8000 tokens in 8 bits, four new ones each (160 MB): 40 us.
#include <hip/hip_runtime.h>

#include "device.h"
#include "kv.h"
#include "kv_device.h"

namespace marlin {
namespace {

using namespace dev;

typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4;
template <int N>
struct Constant {
    static constexpr int value = N;
};
constexpr int kSearch = 6;  // tries to find how large parts are

// Parts of a tile's keys, counted in steps of many rows, in rounds of the four waves' steps of few: at most the root of kRoot times
// as many, as joining takes longer the more there are, and none of less than kLeast.  One sequence, 32 heads over 8 of 128 channels, 16 bits, four
// new tokens: 2000 long 12.7 us (half the root's square 15.0, double 13.0, parts of four rounds 15.0), 20000 long 24.2 (27.0, 30.1 and 24.3); 64 new ones behind
// 8000: 32.5 (half the square 35.2, double 33.5).
struct Many {
    static constexpr int kShift = 2, kLeast = 3, kRoot = 2;  // 16-key tiles of a step (log2)
};
struct Few {
    static constexpr int kShift = 3, kLeast = 2, kRoot = 4;  // of a round
};

__device__ __forceinline__ float16_t mfma32(Elem<_Float16>::vec8 a, Elem<_Float16>::vec8 b, float16_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float16_t mfma32(Elem<__bf16>::vec8 a, Elem<__bf16>::vec8 b, float16_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// A masked key's value may be anything, and its weight of zero does not take an infinity or NaN away.  In steps in which some rows
// do not see all keys what is not finite is left out of the second product, and added by itself for the rows that do see it.
// In the others an infinity becomes NaN where its weight is too small for T: results that are NaN are looked into at the end, until all
// of them are settled (a prompt of 8192 tokens with one NaN among its values 1.4 ms, with nothing else 1.1, without any 0.65 to 0.78).
//
// A dword of elements, or of codes, without those that are not finite.
template <typename T, bool Eight>
__device__ __forceinline__ uint32_t finite_of(uint32_t w)
{
    if constexpr (Eight) {
        const uint32_t odd = ((w & 0x7F7F7F7Fu) + 0x01010101u) >> 7 & 0x01010101u;
        return w & ~(odd * 0xFFu);
    }
    constexpr uint32_t exponent = (__is_same(T, _Float16) ? 0x7C00u : 0x7F80u) * 0x10001u;
    constexpr uint32_t unit = (__is_same(T, _Float16) ? 0x0400u : 0x0080u) * 0x10001u;
    const uint32_t odd = ((w & exponent) + unit) >> 15 & 0x00010001u;
    return w & ~(odd * 0xFFFFu);
}
// One element of the cache, or zero where it is finite.
template <typename T, bool Eight>
__device__ __forceinline__ float odd_at(const void *cache, int64_t at)
{
    float x;
    if constexpr (Eight)
        x = (((const uint8_t *)cache)[at] & 0x7F) == 0x7F ? __builtin_nanf("") : 0.f;
    else
        x = (float)((const T *)cache)[at];
    return __builtin_fabsf(x) < INFINITY ? 0.f : x;
}

// Whether the values of a tile of keys, whose first is at `values`, are not all finite.
template <typename T, int D>
__device__ __forceinline__ bool odd_tile(const T *values, int lane)
{
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < kTileKeys * D / 512; ++i) {
        const u32x4_t w = *(const u32x4_t *)(values + (lane + 64 * i) * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= w[e] ^ finite_of<T, false>(w[e]);
    }
    return __any(odd != 0);
}

// A result that is NaN, and may not be if its row's sum is a number: marked, the first value that is not finite takes its place, others
// are added.  If there is none it stays a NaN.
constexpr uint32_t kMarked = 0x7FC0BEEFu;  // no element becomes this one
__device__ __forceinline__ float marked(float x, bool row) { return row && x != x ? __builtin_bit_cast(float, kMarked) : x; }
__device__ __forceinline__ float add_to_marked(float x, float odd)
{
    return odd == 0.f ? x : __builtin_bit_cast(uint32_t, x) == kMarked ? odd : x + odd;
}
// More values may change it.
__device__ __forceinline__ bool is_open(float x) { return (x == x) | (__builtin_bit_cast(uint32_t, x) == kMarked); }

// The keys that a tile's rows see: those below `sinks` and from a window's lower end on, in tiles of 16 of which the first `sink_tiles`
// and those `skip` further on are taken, 2^shift to a step.
struct Keys {
    int first, last;  // the rows' first and last position
    int end, sinks;   // of what there is, of the sinks below the window
    int sink_tiles, skip, steps;
    // first position of tile t
    __device__ __forceinline__ int position(int t) const { return (t < sink_tiles ? t : t + skip) * kTileKeys; }
};
__device__ __forceinline__ Keys keys_of(const PromptProblem &p, int start, int tokens, int row0, int rows, int shift)
{
    Keys k;
    const int all_rows = tokens * p.group, last_row = (row0 + rows < all_rows ? row0 + rows : all_rows) - 1;
    const int cap = p.width << p.page_shift;
    k.first = start + row0 / p.group;
    k.last = start + last_row / p.group;
    k.end = k.last + 1 < cap ? k.last + 1 : cap;
    if (k.end < 0) k.end = 0;
    int low = 0;
    k.sinks = 0;
    if (p.window) {
        low = k.first >= p.window ? k.first - p.window + 1 : 0;
        k.sinks = p.sinks < low ? p.sinks : low;
    }
    const int all = (k.end + kTileKeys - 1) / kTileKeys, from = low / kTileKeys;
    k.sink_tiles = (k.sinks + kTileKeys - 1) / kTileKeys;
    if (k.sink_tiles > all) k.sink_tiles = all;
    k.skip = (from < all ? from : all) - k.sink_tiles;
    if (k.skip < 0) k.skip = 0;
    k.steps = (all - k.skip + (1 << shift) - 1) >> shift;
    return k;
}

// What a work-group did, for those that join the pieces of tiles whose keys were split: pieces first, first + p.kv_heads ..
struct Record {
    int parts, part, first;  // parts 0: nothing
    int row0, from, tokens;
};
__device__ __forceinline__ Record *record_of(const PromptProblem &p, int index) { return (Record *)p.records + index; }

// What is the same in all lanes, in scalar registers (quotients come from vector ones).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Keys uniform(const Keys &k)
{
    return {uniform(k.first), uniform(k.last), uniform(k.end), uniform(k.sinks), uniform(k.sink_tiles), uniform(k.skip), uniform(k.steps)};
}

// What a work-group does: a tile of rows (tokens from + row / group of a sequence), and which part of its keys.
struct Work {
    int b, from, tokens, start;  // sequence, its first row of q, its new tokens, the first one's position
    int row0;                    // the tile's first row; -1: nothing
    int part, parts, chunk;      // which of its parts, how many there are work-groups for, steps (rounds) of one
    int first;                   // the work-group of the tile's first part; the others' are p.kv_heads apart
};

// The sum over the lanes.
__device__ __forceinline__ float wave_sum(float x)
{
    auto moved = [](float y, auto control, auto rows) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, y), control.value, rows.value, 0xf, true));
    };
    x += moved(x, Constant<0x111>{}, Constant<0xf>{});  // row_shr:1
    x += moved(x, Constant<0x112>{}, Constant<0xf>{});
    x += moved(x, Constant<0x114>{}, Constant<0xf>{});
    x += moved(x, Constant<0x118>{}, Constant<0xf>{});
    x += moved(x, Constant<0x142>{}, Constant<0xa>{});  // row_bcast:15 into rows 1 and 3
    x += moved(x, Constant<0x143>{}, Constant<0xc>{});  // row_bcast:31 into rows 2 and 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// Parts that n steps (rounds) are split into, of `chunk` where they may be as small.
template <typename Kind>
__device__ __forceinline__ int parts_for(int n, int chunk)
{
    if (n <= chunk) return 1;
    int x = (n + chunk - 1) / chunk;
    const int root = (int)__builtin_amdgcn_sqrtf((float)Kind::kRoot * (float)n), most = n / Kind::kLeast;
    if (x > root) x = root;
    if (x > most) x = most;
    return x < 1 ? 1 : x;
}

// The work of one of a kv head's work-groups, found from the sequences' starts and lengths: tiles of `rows` rows, the last of a
// sequence first, as it sees the most, in parts.  A part is as small as it can be with all of them running at once (p.target work-groups):
// 256 new tokens behind 8000 to 30000, four sequences, 32 heads over 8: 395 us, in parts of what all make for each of 512 work-groups 427.
// Where there are as many tiles as that, it is all of a tile.
// 64 sequences are held in the lanes; of more, the waves share the sums.
template <typename Kind>
__device__ __forceinline__ Work find_work(const PromptProblem &p, int rows, int index, int lane, int wave, int *lds_chunks)
{
    const int chunks = (p.B + 63) / 64, head = uniform(index % p.kv_heads), mine = uniform(index / p.kv_heads);
    int held = -1, begin = 0, count = 0, length = 0, tiles = 0, steps = 0;
    auto hold = [&](int at) {
        if (at == held) return;
        held = at;
        const int b = at * 64 + lane;
        begin = count = length = tiles = steps = 0;
        if (b < p.B) {
            begin = p.starts[b];
            int end = p.starts[b + 1];
            begin = begin < 0 ? 0 : begin < p.tokens ? begin : p.tokens;
            end = end < begin ? begin : end < p.tokens ? end : p.tokens;
            count = end - begin;
            length = p.lengths[b];
            if (length < 0) length = 0;
            tiles = (count * p.group + rows - 1) / rows;
            if (p.target > 0 && tiles > 0) steps = keys_of(p, length - count, count, (tiles - 1) * rows, rows, Kind::kShift).steps;
        }
    };
    // two sums over the sequences, in the same order in every work-group
    auto sums_of = [&](auto of) {
        Pair total{0.f, 0.f};
        for (int at = chunks == 1 ? 0 : wave; at < chunks; at += chunks == 1 ? 1 : kWaves) {
            hold(at);
            const Pair x = of();
            total.a += wave_sum(x.a);
            total.b += wave_sum(x.b);
        }
        if (chunks > 1) {
            if (lane == 0) {
                lds_chunks[2 * wave] = __builtin_bit_cast(int, total.a);
                lds_chunks[2 * wave + 1] = __builtin_bit_cast(int, total.b);
            }
            __syncthreads();
            total = {0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                total.a += __builtin_bit_cast(float, lds_chunks[2 * w]);
                total.b += __builtin_bit_cast(float, lds_chunks[2 * w + 1]);
            }
            __syncthreads();
        }
        return Pair{total.a * (float)p.kv_heads, total.b * (float)p.kv_heads};
    };
    int chunk = 1 << 30;
    if (p.target > 0) {
        const float target = (float)p.target;
        const Pair all = sums_of([&] { return Pair{(float)tiles, (float)tiles * (float)steps}; });
        // half of a tile's last part is not there
        const float each = all.b / fmaxf(target - 0.5f * all.a, 0.5f * target);
        if (each < 1e8f) chunk = uniform((int)each + 1);
        for (int i = 0; i < kSearch && chunk < 1 << 28; ++i) {
            const float parts = sums_of([&] { return Pair{(float)tiles * (float)parts_for<Kind>(steps, chunk), 0.f}; }).a;
            if (parts <= target) break;
            const int next = (int)((float)chunk * (parts / target));
            chunk = uniform(next > chunk ? next : chunk + 1);
        }
    }
    int at_chunk = 0, before = 0;
    Work x{0, 0, 0, 0, -1, 0, 1, chunk, 0};
    if (chunks == 1) {
        hold(0);
    } else {
        for (int at = wave; at < chunks; at += kWaves) {
            hold(at);
            const int sum = wave_scan(tiles * parts_for<Kind>(steps, chunk));
            if (lane == 63) lds_chunks[at] = sum;
        }
        __syncthreads();
        at_chunk = -1;
        for (int c0 = 0; c0 < chunks && at_chunk < 0; c0 += 64) {
            const int c = c0 + lane < chunks ? lds_chunks[c0 + lane] : 0, i = wave_scan(c);
            const uint64_t past = __builtin_amdgcn_ballot_w64(before + i > mine);
            const int at = past ? __builtin_ctzll(past) : 63;
            if (past) at_chunk = c0 + at;
            before += __builtin_amdgcn_readlane(i, at) - (past ? __builtin_amdgcn_readlane(c, at) : 0);
        }
        if (at_chunk < 0) return x;
        hold(at_chunk);
    }
    const int parts = parts_for<Kind>(steps, chunk), items = tiles * parts, incl = wave_scan(items);
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + incl > mine);
    if (!past) return x;
    const int at = __builtin_ctzll(past);
    const int n = __builtin_amdgcn_readlane(parts, at), local = mine - before - (__builtin_amdgcn_readlane(incl, at) - __builtin_amdgcn_readlane(items, at));
    x.b = at_chunk * 64 + at;
    x.from = __builtin_amdgcn_readlane(begin, at);
    x.tokens = __builtin_amdgcn_readlane(count, at);
    x.start = __builtin_amdgcn_readlane(length, at) - x.tokens;
    x.part = uniform(local % n);
    x.parts = n;
    x.row0 = uniform((__builtin_amdgcn_readlane(tiles, at) - 1 - local / n) * rows);
    x.first = uniform((mine - x.part) * p.kv_heads + head);
    return x;
}

// Work-groups that share a tile: by its own steps (rounds), which through a window may be more than the last tile's, for which
// work-groups were counted.  0 if those are not all in the launch (starts that are none).
template <typename Kind>
__device__ __forceinline__ int parts_of(const PromptProblem &p, const Work &x, int steps)
{
    int n = parts_for<Kind>(steps, x.chunk);
    n = uniform(n < x.parts ? n : x.parts);
    return n == 1 || (int64_t)x.first + (int64_t)(n - 1) * p.kv_heads < p.groups ? n : 0;
}

// A row's part of what is seen: positions up to `last`, above `above` or below `sinks`.  No branches: what follows from it are
// selects of elements of MFMA results, and the compiler (ROCm 7.2) drops assignments to those in divergent branches.
struct Sight {
    int last, above, sinks;
    __device__ __forceinline__ bool sees(int j) const { return (j <= last) & ((j > above) | (j < sinks)); }
};
__device__ __forceinline__ Sight sight_of(const PromptProblem &p, const Work &t, int row)
{
    const bool have = row < t.tokens * p.group;
    const int pos = have ? t.start + row / p.group : -1;
    return {pos, p.window ? pos - p.window : -1, p.sinks};
}

__device__ __forceinline__ bool is_scale(float s) { return s >= kLeastScale && s <= kMostScale; }

// N tiles of 16 keys of a step as they are loaded: which have pages (bits) and, in an 8-bit cache, their scales.  What follows
// from the scales is found when they are used, a step later, so that nothing waits for them.
template <int N, bool Eight>
struct Raw {
    uint32_t named;
};
template <int N>
struct Raw<N, true> {
    uint32_t named;
    float ks[N], vs[N];
};
// Which tiles are seen at all; and, in an 8-bit cache, factor and summand of their scores and the factor of their weights in the sum.
template <int N, bool Eight>
struct Block {
    uint32_t ok;
};
template <int N>
struct Block<N, true> {
    uint32_t ok;
    float factor[N], add[N], times[N];
};
template <int N>
struct Entries {
    int e[N];
};
// of the tiles of step s
template <int N>
__device__ __forceinline__ Entries<N> load_entries(const PromptProblem &p, const int32_t *table, const Keys &keys, int s)
{
    Entries<N> x;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int pos = keys.position(N * s + u);
        x.e[u] = -1;
        if (pos < keys.end) x.e[u] = scalar_load(table + (pos >> p.page_shift));
    }
    return x;
}
// Pages of a kv head before an entry's (0 for an entry that names no page).
__device__ __forceinline__ int64_t page_head(const PromptProblem &p, int entry, int head)
{
    return (int64_t)((uint32_t)entry < (uint32_t)p.pages ? entry : 0) * p.kv_heads + head;
}
// A position's element in the caches.
__device__ __forceinline__ int64_t place_of(const PromptProblem &p, int entry, int head, int pos, int D)
{
    return ((page_head(p, entry, head) << p.page_shift) + (pos & ((1 << p.page_shift) - 1))) * D;
}
template <int N, bool Eight>
__device__ __forceinline__ Raw<N, Eight> raw_of(const PromptProblem &p, const Entries<N> &x, int head, const Keys &keys, int s)
{
    Raw<N, Eight> k;
    k.named = 0;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        k.named |= ((uint32_t)x.e[u] < (uint32_t)p.pages ? 1u : 0u) << u;
        if constexpr (Eight) {
            const int per_shift = p.page_shift - 4, slot = keys.position(N * s + u) & ((1 << p.page_shift) - 1);
            const float *scale = p.scales + ((page_head(p, x.e[u], head) * 2) << per_shift) + (slot >> 4);
            k.ks[u] = scalar_load(scale);
            k.vs[u] = scalar_load(scale + (1 << per_shift));
        }
    }
    return k;
}
template <int N, bool Eight>
__device__ __forceinline__ Block<N, Eight> block_of(const PromptProblem &p, const Raw<N, Eight> &x)
{
    Block<N, Eight> k;
    k.ok = x.named;
    if constexpr (Eight) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const bool fine = is_scale(x.ks[u]) && is_scale(x.vs[u]);
            if (!fine) k.ok &= ~(1u << u);
            k.factor[u] = fine ? fmaxf(x.ks[u] * p.scale_log2, 0x1p-126f) : 1.f;
            k.add[u] = fine ? __builtin_amdgcn_logf(x.vs[u]) : 0.f;
            k.times[u] = fine ? __builtin_amdgcn_rcpf(x.vs[u]) : 0.f;
        }
    }
    return k;
}
// Eight elements of q, of a row that there is: with the scale's sign, or zero where that is zero.
template <typename V, typename T>
__device__ __forceinline__ V query_of(const PromptProblem &p, const T *q, bool have)
{
    const u32x4_t w = have ? *(const u32x4_t *)q : u32x4_t{};
    return __builtin_bit_cast(V, (w & p.q_and) ^ p.q_xor);
}

// ---- many rows: keys and values through LDS ----

constexpr int kStep = 64;

// Weights are taken against a row's maximum as it was when the results were last brought to it: doing so takes a multiplication of
// every result, and of 32 rows some one's maximum grows by a little in most steps.  float16's weights are times 2^11, 2^15 at the most, those in
// two parts times 2^-4 before they are taken apart.
constexpr float kWideSlack = 4.f;  // log2
template <typename T, bool Two>
constexpr float kWideUnit = !__is_same(T, _Float16) ? 0.f : Two ? -kWideSlack : 11.f;

template <int D>
constexpr int kWideFloats = 64 * kWaves * 4 * ((D / 32) * 4 + 1);

// A wave has 32 rows.  It brings 16 keys of a step, whose page is the same in all lanes, and all waves read all of them.
// K lies in LDS as [key][channel], V^T as [channel][key] with each 16 keys in the order 0-3, 8-11, 4-7, 12-15, rows 16 bytes further
// apart than they are long, an odd number of 16-byte pieces: reads are of distinct banks, and at constant distances.  V^T's
// rows are in an order of their own, eight-channel pieces side by side, so that most writes are too (conflicts take 14 % of
// the LDS's busy cycles, 22 % in an 8-bit cache; an order of the lanes without them took the same time), and a lane's results are whole pieces: row 8 * oct + j of the channels is row j * (D / 8) + oct (96 channels: four-channel pieces, below).
// Two: weights in two parts.
template <typename T, int D, bool Eight, bool Two>
__global__ void __launch_bounds__(64 * kWaves, D <= 128 ? 2 : 1) prompt_kernel(const PromptProblem p)
{
    typedef Elem<T> E;
    typedef typename E::vec8 vec8;
    constexpr int kRows = 32 * kWaves;
    constexpr int kOct = D / 8;                            // eight-channel pieces of a row
    constexpr int kSize = Eight ? 1 : 2;                   // bytes of an element in the cache
    constexpr int kKeyRow = D * 2 + 16, kValueRow = kStep * 2 + 16;  // bytes in LDS
    constexpr int kKeyBytes = kStep * kKeyRow, kValueBytes = D * kValueRow;
    constexpr int kLoad = Eight && D % 64 ? 8 : 16;        // bytes of keys a lane loads at a time
    constexpr int kElems = kLoad / kSize;                  // elements
    constexpr int kKeyPasses = 16 * D / kElems / 64;       // of a wave over its 16 keys
    constexpr int kValueItems = 4 * kOct, kValuePasses = (kValueItems + 63) / 64;  // four keys, eight channels
    constexpr int kPiece = 2 * kSize;                      // dwords of eight elements in the cache
    constexpr int kCt = D / 32, kC = D / 16;
    constexpr float kUnit = kWideUnit<T, Two>;  // log2 of what a weight of 1 is, against a maximum that may be kWideSlack too low
    static_assert(16 * D % (kElems * 64) == 0, "");

    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * (kKeyBytes + kValueBytes)];
    // of a step's four tiles, kept for four steps: whether there is one, whether its values are not all finite, and what its scales
    // make of scores (factor, then add) and of weights in the sum (times)
    struct Info {
        int ok[kWaves], odd[kWaves];
        float factor[kWaves], add[kWaves], times[kWaves];
    };
    __shared__ Info lds_info[4];
    static_assert(sizeof(lds) >= kKvMaxBatch / 64 * 4, "");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int index = p.base + blockIdx.x;
    const int head = uniform(index % p.kv_heads);
    const Work tile = find_work<Many>(p, kRows, index, lane, wave, (int *)lds);
    if (p.target > 0 && tid == 0) record_of(p, index)->parts = 0;
    if (tile.row0 < 0) return;
    const Keys keys = uniform(keys_of(p, tile.start, tile.tokens, tile.row0, kRows, Many::kShift));
    const int parts = parts_of<Many>(p, tile, keys.steps);
    if (tile.part >= parts) return;
    if (parts > 1 && tid == 0) *record_of(p, index) = {parts, tile.part, tile.first, tile.row0, tile.from, tile.tokens};
    const int s0 = uniform((int)((int64_t)keys.steps * tile.part / parts)), s1 = uniform((int)((int64_t)keys.steps * (tile.part + 1) / parts));
    __syncthreads();

    const int32_t *const table = p.table + (int64_t)tile.b * p.table_row;
    auto position_of = [&](int s, int u) { return keys.position(4 * s + u); };  // of a step's tile

    // this lane's row
    const int row = tile.row0 + wave * 32 + col;
    const Sight sight = sight_of(p, tile, row);
    vec8 qf[kC];
    const bool have = row < tile.tokens * p.group;
    const int token = tile.from + (have ? row / p.group : 0), h = head * p.group + (have ? row % p.group : 0);
    const int64_t out_at = have ? (int64_t)token * p.heads + h : -1;
    const T *q = (const T *)p.q + token * p.q_row + h * p.q_head + 8 * half;
#pragma unroll
    for (int c = 0; c < kC; ++c) qf[c] = query_of<vec8>(p, q + 16 * c, have);

    // ---- a step's keys and values: this wave's tile of 16 keys, to registers and from there to LDS ----
    // Keys are a step ahead of values: between a step's weights, which free the scores' registers, and its values' sums come the next one's
    // scores (four chunks in 8 bits 624 us; scores before the weights, in registers of their own, 637; after the sums 623, but heads of 64 and 96 2 % slower).
    uint32_t kreg[kKeyPasses][kLoad / 4], vreg[kValuePasses][4][kPiece];
    const uint32_t key_from = lane * kLoad, value_from = ((lane / kOct) * 4 * D + (lane % kOct) * 8) * kSize;
    // whether every row sees every key of a step, as far as its position says
    auto within = [&](int s) {
        const int t0 = 4 * s, t3 = t0 + 3, last = keys.position(t3);
        bool all = last + kTileKeys - 1 <= keys.first && last + kTileKeys <= keys.end;
        if (p.window) {  // the first tile of the window, the last of the sinks
            const int low = t0 > keys.sink_tiles ? t0 : keys.sink_tiles, sink = t3 < keys.sink_tiles ? t3 : keys.sink_tiles - 1;
            all = all && (low > t3 || keys.position(low) > keys.last - p.window) && (sink < t0 || keys.position(sink) + kTileKeys <= p.sinks);
        }
        return all;
    };
    // this wave's tile of a step: its page's entry, where it lies (bytes), whether there is one, its scales
    struct Mine {
        int64_t at;
        bool named;
        bool within;
        float ks, vs;
    };
    auto entry_of = [&](int s) {
        const int pos = position_of(s, wave);
        int e = -1;
        if (s < s1 && pos < keys.end) e = scalar_load(table + (pos >> p.page_shift));
        return e;
    };
    auto load_keys = [&](int s, int entry) {
        Mine x;
        entry = __builtin_amdgcn_readfirstlane(entry);
        x.named = (uint32_t)entry < (uint32_t)p.pages;
        x.within = within(s);
        const int pos = position_of(s, wave);
        x.at = place_of(p, entry, head, pos, D) * kSize;
        if constexpr (Eight) {
            const int per_shift = p.page_shift - 4, slot = pos & ((1 << p.page_shift) - 1);
            const float *scale = p.scales + ((page_head(p, entry, head) * 2) << per_shift) + (slot >> 4);
            x.ks = scalar_load(scale);
            x.vs = scalar_load(scale + (1 << per_shift));
        }
        if (x.named) {
            const uint8_t *const k = (const uint8_t *)p.k + x.at;
#pragma unroll
            for (int i = 0; i < kKeyPasses; ++i)
                __builtin_memcpy(kreg[i], __builtin_assume_aligned(k + key_from + i * 64 * kLoad, kLoad), kLoad);
        }
        return x;
    };
    auto load_values = [&](const Mine &x) {
        if (!x.named) return;
        const uint8_t *const v = (const uint8_t *)p.v + x.at;
#pragma unroll
        for (int i = 0; i < kValuePasses; ++i)
            if (kValueItems % 64 == 0 || lane + 64 * i < kValueItems) {
                static_assert(kValuePasses == 1 || 64 % kOct == 0, "");
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    __builtin_memcpy(vreg[i][j], __builtin_assume_aligned(v + value_from + (i * (64 / kOct) * 4 + j) * D * kSize, 8 * kSize), 8 * kSize);
            }
    };
    auto is_fine = [&](const Mine &x) {
        if constexpr (Eight) return x.named && is_scale(x.ks) && is_scale(x.vs);
        return x.named;
    };
    auto store_keys = [&](int s, const Mine &x) {
        uint8_t *const to = lds + (s & 1) * kKeyBytes;
        const bool fine = is_fine(x);
        if (lane == 0) {
            Info &info = lds_info[s & 3];
            info.ok[wave] = fine;
            if constexpr (Eight) {
                info.factor[wave] = fine ? fmaxf(x.ks * p.scale_log2, 0x1p-126f) : 1.f;
                info.add[wave] = fine ? __builtin_amdgcn_logf(x.vs) : 0.f;
                info.times[wave] = fine ? __builtin_amdgcn_rcpf(x.vs) : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < kKeyPasses; ++i) {
            const int n = (lane + 64 * i) * kElems, key = kTileKeys * wave + n / D, ch = n % D;
#pragma unroll
            for (int j = 0; j < kElems / 8; ++j) {
                vec8 y;
                if constexpr (Eight)
                    y = E::of_codes(kreg[i][2 * j], kreg[i][2 * j + 1]);
                else
                    __builtin_memcpy(&y, kreg[i], 16);
                *(vec8 *)(to + key * kKeyRow + (ch + 8 * j) * 2) = y;
            }
        }
    };
    auto store_values = [&](int s, const Mine &x) {
        if (!(x.within && is_fine(x))) {
            const int pos = position_of(s, wave);
            // what no row sees is zero; of the rest what is finite
            uint32_t odd = 0;
#pragma unroll
            for (int i = 0; i < kValuePasses; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool seen = x.named & (pos + ((lane + 64 * i) / kOct) * 4 + j < keys.end);
#pragma unroll
                    for (int w = 0; w < kPiece; ++w) {
                        const uint32_t y = seen ? vreg[i][j][w] : 0, z = finite_of<T, Eight>(y);
                        odd |= y ^ z;
                        vreg[i][j][w] = z;
                    }
                }
            const bool any = __any((kValueItems % 64 == 0 || lane < kValueItems) & (odd != 0));
            if (lane == 0) lds_info[s & 3].odd[wave] = any;
        }
        uint8_t *const to_values = lds + 2 * kKeyBytes + (s & 1) * kValueBytes;
#pragma unroll
        for (int i = 0; i < kValuePasses; ++i) {
            if (kValueItems % 64 == 0 || lane + 64 * i < kValueItems) {
                const int quad = (lane + 64 * i) / kOct, oct = (lane + 64 * i) % kOct;
                uint8_t *const to = to_values + (2 * wave + (quad & 1)) * 16 + (quad >> 1) * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    uint32_t w[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if constexpr (Eight)
                            w[h] = E::of_two_codes(__builtin_amdgcn_perm(vreg[i][2 * h + 1][j >> 2], vreg[i][2 * h][j >> 2],
                                                                         (j & 2) ? 0x07030602u : 0x05010400u), j & 1);
                        else
                            w[h] = __builtin_amdgcn_perm(vreg[i][2 * h + 1][j >> 1], vreg[i][2 * h][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
                    }
                    // channel 8 oct + j; with 96 of them the fours are side by side, by eight of them
                    const int four = 2 * oct + (j >> 2), row = D == 96 ? 32 * (four >> 3) + 8 * (j & 3) + (four & 7) : j * kOct + oct;
                    __builtin_memcpy(__builtin_assume_aligned(to + row * kValueRow, 8), w, 8);
                }
            }
        }
    };
    // the channel of element i of accumulator ct
    auto channel_of = [&](int ct, int i) {
        if (D == 96) return 4 * (8 * ct + 4 * half + (i & 3)) + (i >> 2);
        const int row = 32 * ct + 8 * (i >> 2) + (i & 3);
        return 8 * (row % kOct) + row / kOct + 32 * half;
    };

    float16_t acc[kCt];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int ct = 0; ct < kCt; ++ct) acc[ct] = float16_t{};

    typedef float16_t scores_t[2];
    const uint32_t key_at = col * kKeyRow + half * 16, value_at = 2 * kKeyBytes + col * kValueRow + half * 16;
    auto score = [&](int s, scores_t &x) {
        const uint8_t *const from = lds + (s & 1) * kKeyBytes + key_at;
        x[0] = x[1] = float16_t{};
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const vec8 a = *(const vec8 *)(from + 32 * kt * kKeyRow + c * 32);
                x[kt] = mfma32(a, qf[c], x[kt]);
            }
    };
    // which of a step's tiles are there
    auto ok_of = [&](int s) { return (uint32_t)__builtin_amdgcn_ballot_w64(lds_info[s & 3].ok[lane & 3] != 0) & 15u; };
    // scores that are not seen, then the maximum (of what the factors make of them) with the sums brought to it
    auto look = [&](int s, bool inside, scores_t &x, float &top) {
        const uint32_t ok = ok_of(s);
        if (!(inside && ok == 15u)) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = position_of(s, 2 * kt + (i >> 3)) + 8 * ((i >> 2) & 1) + 4 * half + (i & 3);
                    const bool seen = ((ok >> (2 * kt + (i >> 3)) & 1) != 0) & sight.sees(j) & (j < keys.end);
                    x[kt][i] = seen ? x[kt][i] : -INFINITY;
                }
        }
        float t = m;
        if constexpr (Eight) {
            const Info &info = lds_info[s & 3];
#pragma unroll
            for (int g16 = 0; g16 < 4; ++g16) {
                float y = x[g16 >> 1][8 * (g16 & 1)];
#pragma unroll
                for (int e = 1; e < 8; ++e) y = fmaxf(y, x[g16 >> 1][8 * (g16 & 1) + e]);
                t = fmaxf(t, __builtin_fmaf(y, info.factor[g16], info.add[g16]));
            }
        } else {
            float y = x[0][0];
#pragma unroll
            for (int e = 1; e < 32; ++e) y = fmaxf(y, x[e >> 4][e & 15]);
            t = fmaxf(t, y * p.scale_log2);
        }
        const Pair halves = exchange<32>(t);
        top = fmaxf(halves.a, halves.b);
    };
    auto rescale = [&](float top) {
        // the maximum that weights are taken against moves only where it is more than the slack too low
        const bool moves = top > m + kWideSlack;
        if (__any(moves)) {
            const float to = moves ? top : m, keep = moves ? __builtin_amdgcn_exp2f(m - to) : 1.f;
            l *= keep;
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct) acc[ct] *= keep;
            m = to;
        }
    };
    constexpr int kParts = Two ? 2 : 1;
    typedef vec8 weights_t[kParts][4];
    auto weigh = [&](int s, const scores_t &x, weights_t &weights) {
        const float unit = kUnit - (m == -INFINITY ? 0.f : m);
#pragma unroll
        for (int g16 = 0; g16 < 4; ++g16) {
            float f = p.scale_log2, add = unit, sum = 0.f;
            if constexpr (Eight) {
                f = lds_info[s & 3].factor[g16];
                add += lds_info[s & 3].add[g16];
            }
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(x[g16 >> 1][8 * (g16 & 1) + e], f, add));
                const float z = __builtin_amdgcn_exp2f(__builtin_fmaf(x[g16 >> 1][8 * (g16 & 1) + e + 1], f, add));
                sum += y + z;
                if constexpr (Two) {
                    const typename E::Parts both = E::part(y, z);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        weights[0][g16][e + i] = both.first[i];
                        weights[kParts - 1][g16][e + i] = both.rest[i];
                    }
                } else {
                    weights[0][g16][e] = (T)y;
                    weights[0][g16][e + 1] = (T)z;
                }
            }
            if constexpr (Eight) sum *= lds_info[s & 3].times[g16];
            l += sum;
        }
    };
    auto add_values = [&](int s, const weights_t &weights) {
        const uint8_t *const from = lds + (s & 1) * kValueBytes + value_at;
#pragma unroll
        for (int g16 = 0; g16 < 4; ++g16)
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct) {
                const vec8 a = *(const vec8 *)(from + 32 * ct * kValueRow + g16 * 32);
#pragma unroll
                for (int part = 0; part < kParts; ++part) acc[ct] = mfma32(a, weights[part][g16], acc[ct]);
            }
    };
    // values of a step that are not finite, where some rows do not see all keys
    auto add_odd = [&](int s, bool inside) {
        const uint32_t ok = ok_of(s);
        if (inside && ok == 15u) return;
        // a wave whose tile every row sees has not looked
        uint32_t odd = (uint32_t)__builtin_amdgcn_ballot_w64(lds_info[s & 3].odd[lane & 3] != 0) & 15u;
        if (inside) odd &= ~ok;
        if (odd == 0) return;
#pragma unroll 1
        for (int n = 0; n < kStep; ++n) {
            const int j = position_of(s, n >> 4) + (n & 15);
            if (!(ok >> (n >> 4) & 1) || j >= keys.end) continue;
            const int64_t at = place_of(p, scalar_load(table + (j >> p.page_shift)), head, j, D);
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = odd_at<T, Eight>(p.v, at + channel_of(ct, i));
                    acc[ct][i] += sight.sees(j) ? x : 0.f;
                }
        }
    };

    if (s0 < s1) {
        scores_t x;
        weights_t weights;
        float top;
        int entry = entry_of(s0 + 1);
        Mine values = load_keys(s0, entry_of(s0)), next = values;  // of the step whose values are to come next; of the one after it
        store_keys(s0, values);
        load_values(values);
        next = load_keys(s0 + 1, entry);
        entry = entry_of(s0 + 2);
        __syncthreads();
        score(s0, x);
        bool inside = values.within;  // of the step at hand
        look(s0, inside, x, top);
        rescale(top);
        store_values(s0, values);
        store_keys(s0 + 1, next);
#pragma unroll 1
        for (int s = s0; s + 1 < s1; ++s) {
            __syncthreads();
            values = next;
            load_values(values);
            next = load_keys(s + 2, entry);
            entry = entry_of(s + 3);
            weigh(s, x, weights);
            score(s + 1, x);
            add_values(s, weights);
            look(s + 1, values.within, x, top);
            add_odd(s, inside);
            inside = values.within;
            rescale(top);
            store_values(s + 1, values);
            store_keys(s + 2, next);
        }
        __syncthreads();
        weigh(s1 - 1, x, weights);
        add_values(s1 - 1, weights);
        add_odd(s1 - 1, inside);
    }
    const Pair halves = exchange<32>(l);
    l = halves.a + halves.b;
    if constexpr (!Eight) {  // codes have no infinities
        float sum = 0.f;
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += acc[ct][i];
        if (__any((sum != sum) & (l == l))) {
#pragma unroll
            for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[ct][i] = marked(acc[ct][i], l == l);
#pragma unroll 1
            for (int t = 4 * s0; t < 4 * s1; ++t) {
                const int pos = keys.position(t);
                if (pos >= keys.end) break;
                const int entry = scalar_load(table + (pos >> p.page_shift));
                if ((uint32_t)entry >= (uint32_t)p.pages) continue;
                const int64_t first = place_of(p, entry, head, pos, D);
                if (!odd_tile<T, D>((const T *)p.v + first, lane)) continue;
#pragma unroll 1
                for (int j = pos; j < pos + kTileKeys && j < keys.end; ++j)
#pragma unroll
                    for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float x = odd_at<T, Eight>(p.v, first + (j - pos) * D + channel_of(ct, i));
                            acc[ct][i] = add_to_marked(acc[ct][i], sight.sees(j) ? x : 0.f);
                        }
                bool open = false;
#pragma unroll
                for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
                    for (int i = 0; i < 16; ++i) open |= is_open(acc[ct][i]);
                if (!__any(open & have)) break;
            }
        }
    }

    // ---- a part of the tile's keys: left for the joining kernel ----
    if (parts > 1) {
        float4_t *const slot = (float4_t *)(p.partials + (int64_t)index * kWideFloats<D>) + lane;
        constexpr int kPer = kCt * 4 + 1;  // blocks of 64 float4 of a wave
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                slot[(wave * kPer + ct * 4 + q) * 64] =
                    float4_t{acc[ct][4 * q], acc[ct][4 * q + 1], acc[ct][4 * q + 2], acc[ct][4 * q + 3]};
        slot[(wave * kPer + kCt * 4) * 64] = float4_t{m, l, 0.f, 0.f};
        return;
    }

    // ---- the finished row: a lane holds pieces of eight channels (96: of four) ----
    if (out_at < 0) return;
    const float inv = 1.f / (Two ? l * E::kWeightUnit : l);
    T *const to = (T *)p.out + out_at * D;
    auto result = [&](int ct, int i) { return l == 0.f ? (T)0.f : (T)(acc[ct][i] * inv); };
    constexpr int kPieces = D == 96 ? 12 : D / 16, kChannels = D == 96 ? 4 : 8;  // a lane's
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
        T y[kChannels];
#pragma unroll
        for (int j = 0; j < kChannels; ++j) {
            // D = 96: four 8 ct + 4 half + i, its channels in q = j; else piece 8 (n / 4) + 4 half + n % 4, channel j in row j * kOct + piece
            const int row = j * kOct + 8 * (n >> 2) + (n & 3);
            y[j] = D == 96 ? result(n >> 2, 4 * j + (n & 3)) : result(row >> 5, 4 * ((row & 31) >> 3) + (n & 3));
        }
        __builtin_memcpy(__builtin_assume_aligned(to + kChannels * (8 * (n >> 2) + 4 * half + (n & 3)), 2 * kChannels), y, 2 * kChannels);
    }
    if (p.lse && half == 0) p.lse[out_at] = (m + __builtin_amdgcn_logf(l) - kUnit) * 0.693147180559945f;
}

// ---- few rows: keys and values straight to registers, the waves share the keys ----

template <int D, int RT>
constexpr int kFewFloats = 64 * 4 * RT * (D / 16 + 1);

// RT: 16-row columns of the tile.  A wave takes steps of 32 keys as the kernel of one token per sequence does (attend.hip), with the
// rows for its heads.
template <typename T, int D, int RT, bool Eight>
__global__ void __launch_bounds__(64 * kWaves, D > 128 ? 1 : 2) prompt_few_kernel(const PromptProblem p)
{
    typedef Elem<T> E;
    typedef typename E::vec8 vec8;
    constexpr int kRows = 16 * RT, KT = 2, kKeys = 32;
    constexpr int kQ = D / 32;
    constexpr int kHalves = D > 128 && !Eight ? 2 : 1;
    constexpr int kCh = D / 16 / kHalves;
    constexpr int kValueDw = Eight ? (kCh + 3) / 4 : kCh / 2;
    constexpr bool kBy32 = D % 64 != 0;
    constexpr int kKeyDw = Eight ? D / 16 : kQ * 4;
    constexpr int kAcc = D / 16;
    constexpr int kSlot = kFewFloats<D, RT>;
    // Values are read past the caches where rows are whole lines of 128 bytes and a sequence has 16 rows at the most on the average, which where all are
    // alike is one tile: 100 sequences of 5000 tokens, four new ones each, 8 bits 212 us, through the caches 230, in 16 bits 359 and 390 (keys too: of
    // 200 sequences 190 for 184).  A sequence of more rows than that reads its values once for each tile: one and seven new ones in turn 219 and
    // 214, in 16 bits 385 and 370; one three times, then thirteen 247 and 238, 423 and 392.  Two tiles a sequence, 48 rows: 57 so, 54 through the caches.
    constexpr bool kOnce = RT == 1 && D * (Eight ? 1 : 2) % 128 == 0;

    __shared__ float4_t lds_acc[kWaves][kAcc][64];
    __shared__ float lds_m[kWaves][kHeadTile], lds_l[kWaves][kHeadTile];
    static_assert(sizeof(lds_acc) >= kKvMaxBatch / 64 * 4, "");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int index = p.base + blockIdx.x;
    const int head = uniform(index % p.kv_heads);
    const Work tile = find_work<Few>(p, kRows, index, lane, wave, (int *)&lds_acc[0][0][0]);
    if (p.target > 0 && tid == 0) record_of(p, index)->parts = 0;
    if (tile.row0 < 0) return;
    const Keys keys = uniform(keys_of(p, tile.start, tile.tokens, tile.row0, kRows, 1));
    const int rounds = (keys.steps + kWaves - 1) / kWaves, parts = parts_of<Few>(p, tile, rounds);
    if (tile.part >= parts) return;
    if (parts > 1 && tid == 0) *record_of(p, index) = {parts, tile.part, tile.first, tile.row0, tile.from, tile.tokens};
    const int s0 = uniform((int)((int64_t)rounds * tile.part / parts)) * kWaves, last = uniform((int)((int64_t)rounds * (tile.part + 1) / parts)) * kWaves;
    const int s1 = last < keys.steps ? last : keys.steps;
    __syncthreads();

    const int32_t *const table = p.table + (int64_t)tile.b * p.table_row;
    auto position_of = [&](int s, int u) { return keys.position(2 * s + u); };  // of a step's tile
    Sight sight[RT];
    vec8 qf[RT][kQ];
    int64_t out_at[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = tile.row0 + rt * 16 + r;
        sight[rt] = sight_of(p, tile, row);
        const bool have = row < tile.tokens * p.group;
        const int token = tile.from + (have ? row / p.group : 0), h = head * p.group + (have ? row % p.group : 0);
        out_at[rt] = have ? (int64_t)token * p.heads + h : -1;
        const T *q = (const T *)p.q + token * p.q_row + h * p.q_head;
#pragma unroll
        for (int t = 0; t < kQ; ++t) qf[rt][t] = query_of<vec8>(p, Eight && !kBy32 ? q + 16 * g + 64 * (t >> 1) + 8 * (t & 1) : q + 8 * g + 32 * t, have);
    }

    uint32_t kf[KT][kKeyDw] = {}, vr[KT][4][kHalves][kValueDw] = {};
    struct Places {
        int64_t at[KT];
    };
    auto places_of = [&](const Entries<KT> &x, int s) {
        Places k;
#pragma unroll
        for (int u = 0; u < KT; ++u) k.at[u] = place_of(p, x.e[u], head, position_of(s, u), D);
        return k;
    };
    // of tiles without a page the registers keep what they hold, which is masked
    auto load_keys = [&](const Places &k, uint32_t named) {
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            if (!(named >> u & 1)) continue;
            if constexpr (!Eight) {
                const T *from = (const T *)p.k + k.at[u] + (r * D + 8 * g);
#pragma unroll
                for (int t = 0; t < kQ; ++t) __builtin_memcpy(&kf[u][4 * t], __builtin_assume_aligned(from + 32 * t, 16), 16);
            } else {
                constexpr int kPiece = kBy32 ? 8 : 16;
                const uint8_t *from = (const uint8_t *)p.k + k.at[u] + r * D;
#pragma unroll
                for (int t = 0; t < D / (4 * kPiece); ++t)
                    __builtin_memcpy(&kf[u][kPiece / 4 * t], __builtin_assume_aligned(from + kPiece * (g + 4 * t), kPiece), kPiece);
            }
        }
    };
    auto load_values = [&](const Places &k, uint32_t named) {
        auto read = [](uint32_t(&to)[kValueDw], const void *from) {
            if constexpr (kOnce)
                load_dwords_once<kValueDw>(to, from);
            else
                load_dwords<kValueDw>(to, from);
        };
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            if (!(named >> u & 1)) continue;
            if constexpr (!Eight) {
                const T *v = (const T *)p.v + k.at[u] + (4 * g * D + kCh * r);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf) read(vr[u][i][hf], v + i * D + 128 * hf);
            } else {
                const uint8_t *v = (const uint8_t *)p.v + k.at[u] + 4 * g * D;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (kBy32) {
                        vr[u][i][0][0] = *(const uint32_t *)(v + i * D + 4 * r);
                        vr[u][i][0][1] = *(const uint16_t *)(v + i * D + 64 + 2 * r);
                    } else {
                        read(vr[u][i][0], v + i * D + kCh * r);
                    }
                }
            }
        }
    };
    float4_t acc[RT][kAcc];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.f;
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc[rt][j] = float4_t{0.f, 0.f, 0.f, 0.f};
    }
    // the channel that row x of accumulator j stands for
    auto channel_of = [](int j, int x) {
        return Eight && kBy32 ? (j < 4 ? 4 * x + j : 60 + 2 * x + j) : 128 * (j / kCh) + kCh * x + j % kCh;
    };
    // four keys' elements of channel piece hf, j of both tiles, as the second product's operand
    auto values_of = [&](int hf, int j) -> vec8 {
        u32x4_t w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (Eight)
                w[e] = E::of_two_codes(__builtin_amdgcn_perm(vr[e >> 1][2 * (e & 1) + 1][hf][j >> 2], vr[e >> 1][2 * (e & 1)][hf][j >> 2],
                                                             (j & 2) ? 0x07030602u : 0x05010400u), j & 1);
            else
                w[e] = __builtin_amdgcn_perm(vr[e >> 1][2 * (e & 1) + 1][hf][j >> 1], vr[e >> 1][2 * (e & 1)][hf][j >> 1],
                                             (j & 1) ? 0x07060302u : 0x05040100u);
        }
        return __builtin_bit_cast(vec8, w);
    };

    int s = s0 + wave;
    if (s < s1) {
        const Entries<KT> first = load_entries<KT>(p, table, keys, s);
        Raw<KT, Eight> raw = raw_of<KT, Eight>(p, first, head, keys, s), next = raw;
        Places places = places_of(first, s);
        load_keys(places, raw.named);
        load_values(places, raw.named);
        Entries<KT> ahead{};
        if (s + kWaves < s1) ahead = load_entries<KT>(p, table, keys, s + kWaves);
#pragma unroll 1
        while (true) {
            float4_t sc[RT][KT];
#pragma unroll
            for (int u = 0; u < KT; ++u) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) sc[rt][u] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < kQ; ++t) {
                    vec8 x;
                    if constexpr (Eight)
                        x = E::of_codes(kf[u][2 * t], kf[u][2 * t + 1]);
                    else
                        __builtin_memcpy(&x, &kf[u][4 * t], 16);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) sc[rt][u] = E::mfma(x, qf[rt][t], sc[rt][u]);
                }
            }
            const int pos[KT] = {position_of(s, 0), position_of(s, 1)};
            const bool more = s + kWaves < s1;
            issue_order_point();
            if (more) {
                next = raw_of<KT, Eight>(p, ahead, head, keys, s + kWaves);
                places = places_of(ahead, s + kWaves);
                load_keys(places, next.named);
                if (s + 2 * kWaves < s1) ahead = load_entries<KT>(p, table, keys, s + 2 * kWaves);
            }
            const Block<KT, Eight> cur = block_of<KT, Eight>(p, raw);
            bool all = cur.ok == 3u && pos[1] + kTileKeys - 1 <= keys.first && pos[1] + kTileKeys <= keys.end;
            if (p.window) {
#pragma unroll
                for (int u = 0; u < KT; ++u) all = all && (pos[u] > keys.last - p.window || pos[u] + kTileKeys <= p.sinks);
            }
            if (!all) {  // what no row sees: zero
#pragma unroll
                for (int u = 0; u < KT; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(cur.ok >> u & 1) || pos[u] + 4 * g + i >= keys.end) {
#pragma unroll
                            for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                                for (int w = 0; w < kValueDw; ++w) vr[u][i][hf][w] = 0;
                        }
            }
            vec8 weights[RT], rest[RT];  // in two parts
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
                for (int u = 0; u < KT; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (Eight)
                            sc[rt][u][i] = __builtin_fmaf(sc[rt][u][i], cur.factor[u], cur.add[u]);
                        else
                            sc[rt][u][i] *= p.scale_log2;
                    }
                if (!all) {
#pragma unroll
                    for (int u = 0; u < KT; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int j = pos[u] + 4 * g + i;
                            const bool seen = ((cur.ok >> u & 1) != 0) & sight[rt].sees(j) & (j < keys.end);
                            sc[rt][u][i] = seen ? sc[rt][u][i] : -INFINITY;
                        }
                }
                float top = m[rt];
#pragma unroll
                for (int u = 0; u < KT; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[rt][u][i]);
                top = max_over_groups(top);
                const float ref = top == -INFINITY ? 0.f : top;
                if (__any(top > m[rt])) {
                    const float keep = __builtin_amdgcn_exp2f(m[rt] - ref);
                    l[rt] *= keep;
#pragma unroll
                    for (int j = 0; j < kAcc; ++j) acc[rt][j] *= keep;
                }
                m[rt] = top;
#pragma unroll
                for (int u = 0; u < KT; ++u) {
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        const float x = __builtin_amdgcn_exp2f(sc[rt][u][i] - ref), y = __builtin_amdgcn_exp2f(sc[rt][u][i + 1] - ref);
                        sum += x + y;
                        const typename E::Parts both = E::part(x, y);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            weights[rt][4 * u + i + e] = both.first[e];
                            rest[rt][4 * u + i + e] = both.rest[e];
                        }
                    }
                    if constexpr (Eight) sum *= cur.times[u];
                    l[rt] += sum;
                }
            }
            if (!all) {
                uint32_t odd = 0;
#pragma unroll
                for (int u = 0; u < KT; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                            for (int w = 0; w < kValueDw; ++w) {
                                const uint32_t x = finite_of<T, Eight>(vr[u][i][hf][w]);
                                odd |= x ^ vr[u][i][hf][w];
                                vr[u][i][hf][w] = x;
                            }
                if (__any(odd != 0)) {
#pragma unroll 1
                    for (int n = 0; n < kKeys; ++n) {
                        const int j = position_of(s, n >> 4) + (n & 15);
                        if (!(cur.ok >> (n >> 4) & 1) || j >= keys.end) continue;
                        const int64_t at = place_of(p, scalar_load(table + (j >> p.page_shift)), head, j, D);
#pragma unroll
                        for (int c = 0; c < kAcc; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float x = odd_at<T, Eight>(p.v, at + channel_of(c, 4 * g + i));
#pragma unroll
                                for (int rt = 0; rt < RT; ++rt) acc[rt][c][i] += sight[rt].sees(j) ? x : 0.f;
                            }
                    }
                }
            }
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                for (int j = 0; j < kCh; ++j) {
                    const vec8 x = values_of(hf, j);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        acc[rt][hf * kCh + j] = E::mfma(x, weights[rt], acc[rt][hf * kCh + j]);
                        acc[rt][hf * kCh + j] = E::mfma(x, rest[rt], acc[rt][hf * kCh + j]);
                    }
                }
            issue_order_point();
            if (!more) break;
            load_values(places, next.named);
            raw = next;
            s += kWaves;
        }
    }
    if constexpr (!Eight) {
        bool look = false;
        float of_row[RT];  // the row's sum
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            of_row[rt] = sum_over_groups(l[rt]);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < kAcc; ++j) sum += (acc[rt][j][0] + acc[rt][j][1]) + (acc[rt][j][2] + acc[rt][j][3]);
            look |= (sum != sum) & (of_row[rt] == of_row[rt]);
        }
        if (__any(look)) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int j = 0; j < kAcc; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[rt][j][i] = marked(acc[rt][j][i], of_row[rt] == of_row[rt]);
#pragma unroll 1
            for (int t = KT * (s0 + wave); t < KT * s1; t += t % KT + 1 < KT ? 1 : KT * (kWaves - 1) + 1) {
                const int pos = keys.position(t);
                if (pos >= keys.end) break;
                const int entry = scalar_load(table + (pos >> p.page_shift));
                if ((uint32_t)entry >= (uint32_t)p.pages) continue;
                const int64_t first = place_of(p, entry, head, pos, D);
                if (!odd_tile<T, D>((const T *)p.v + first, lane)) continue;
#pragma unroll 1
                for (int j = pos; j < pos + kTileKeys && j < keys.end; ++j)
#pragma unroll
                    for (int c = 0; c < kAcc; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = odd_at<T, Eight>(p.v, first + (j - pos) * D + channel_of(c, 4 * g + i));
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt) acc[rt][c][i] = add_to_marked(acc[rt][c][i], sight[rt].sees(j) ? x : 0.f);
                        }
                bool open = false;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int c = 0; c < kAcc; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) open |= is_open(acc[rt][c][i]) & (out_at[rt] >= 0);
                if (!__any(open)) break;
            }
        }
    }

    // ---- the waves' pieces; a part of the tile's keys is left for the joining kernel ----
    float *const slot = p.partials + (int64_t)index * kSlot;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kAcc; ++j) lds_acc[wave][j][lane] = acc[rt][j];
        const float sum_l = sum_over_groups(l[rt]);
        if (g == 0) {
            lds_m[wave][r] = m[rt];
            lds_l[wave][r] = sum_l;
        }
        __syncthreads();
        float top = -INFINITY, sum = 0.f, f[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds_m[w][r]);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            f[w] = __builtin_amdgcn_exp2f(lds_m[w][r] - ref);
            sum += lds_l[w][r] * f[w];
        }
        const float inv = 1.f / (sum * E::kWeightUnit);
#pragma unroll 1
        for (int j = wave; j < kAcc; j += kWaves) {
            float4_t o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) o += lds_acc[w][j][lane] * f[w];
            if (parts > 1) {
                ((float4_t *)slot)[(rt * (kAcc + 1) + j) * 64 + lane] = o;
                if (j == 0) ((float4_t *)slot)[(rt * (kAcc + 1) + kAcc) * 64 + lane] = float4_t{top, sum, 0.f, 0.f};
                continue;
            }
            if (out_at[rt] < 0) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) ((T *)p.out)[out_at[rt] * D + channel_of(j, 4 * g + i)] = sum == 0.f ? (T)0.f : (T)(o[i] * inv);
            if (p.lse && g == 0 && j == 0) p.lse[out_at[rt]] = (top + __builtin_amdgcn_logf(sum)) * 0.693147180559945f;
        }
    }
}

// ---- pieces of tiles whose keys were split ----

// A piece is blocks of 64 float4, kBlocks of a lane's results and one of its row's maximum and sum, RT times of each wave.  The
// work-groups that made a tile's pieces join a share of its blocks each: few pieces a wave a block, in order; of many
// the waves take some each, in order, and are added up in LDS.  So the pieces of any number are read side by side, and the
// same bits come of them every time.
template <typename T, int D, int RT, bool Few, bool Eight, bool Two>
__global__ void __launch_bounds__(64 * kWaves) prompt_join_kernel(const PromptProblem p)
{
    constexpr int kBlocks = Few ? D / 16 : D / 8;  // of a wave's rows
    constexpr int kAll = (Few ? 1 : kWaves) * RT * kBlocks;
    constexpr int kFloats = Few ? kFewFloats<D, RT> : kWideFloats<D>;
    constexpr int kHalves = D > 128 && !Eight ? 2 : 1, kCh = D / 16 / kHalves, kOct = D / 8;
    // what the sum is times (log2), and results beside it
    constexpr float kUnit = Few ? 0.f : kWideUnit<T, Two>, kWeight = Two ? Elem<T>::kWeightUnit : 1.f;
    __shared__ float4_t lds_o[kWaves][64];
    __shared__ float lds_top[kWaves][64], lds_sum[kWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int index = p.base + blockIdx.x, head = uniform(index % p.kv_heads);
    const Record x = *record_of(p, index);
    const int parts = uniform(x.parts), part = uniform(x.part);
    if (parts == 0) return;
    const float4_t *const pieces = (const float4_t *)(p.partials + (int64_t)x.first * kFloats) + lane;
    const int64_t stride = (int64_t)p.kv_heads * kFloats / 4;
    const int from = kAll * part / parts, to = kAll * (part + 1) / parts;
    // pieces k0, k0 + step .. of a block: their results added up, brought to their maximum; eight under way together
    struct Joined {
        float top, sum;
        float4_t y;
    };
    auto join = [&](const float4_t *ml, const float4_t *o, int k0, int step) {
        Joined x{-INFINITY, 0.f, float4_t{0.f, 0.f, 0.f, 0.f}};
        constexpr int kAhead = 8;
#pragma unroll 1
        for (int k = k0; k < parts; k += kAhead * step) {
            float4_t v[kAhead], z[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const bool have = k + i * step < parts;  // or the first again, as nothing: a weight of zero does not take an infinity away
                const int64_t at = (have ? k + i * step : k) * stride;
                v[i] = ml[at];
                z[i] = o[at];
                v[i][0] = have ? v[i][0] : -INFINITY;
#pragma unroll
                for (int e = 0; e < 4; ++e) z[i][e] = have ? z[i][e] : 0.f;
            }
            float top = x.top;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) top = fmaxf(top, v[i][0]);
            const float ref = top == -INFINITY ? 0.f : top, keep = __builtin_amdgcn_exp2f(x.top - ref);
            x.top = top;
            x.sum *= keep;
            x.y *= keep;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const float f = __builtin_amdgcn_exp2f(v[i][0] - ref);
                x.sum += v[i][1] * f;
                x.y += z[i] * f;
            }
        }
        return x;
    };
    auto write = [&](int group, int j, float top, float sum, float4_t y) {
        const int row = x.row0 + (Few ? group * 16 + (lane & 15) : group * 32 + (lane & 31));
        if (row >= x.tokens * p.group) return;
        const int64_t at = (int64_t)(x.from + row / p.group) * p.heads + head * p.group + row % p.group;
        const float inv = 1.f / (sum * kWeight);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int ch;
            if constexpr (Few) {
                const int c = 4 * (lane >> 4) + i;
                ch = Eight && D % 64 ? (j < 4 ? 4 * c + j : 60 + 2 * c + j) : 128 * (j / kCh) + kCh * c + j % kCh;
            } else {
                const int r = 32 * (j >> 2) + 8 * (j & 3) + 4 * (lane >> 5) + i;
                ch = D == 96 ? 4 * (8 * (j >> 2) + 4 * (lane >> 5) + i) + (j & 3) : 8 * (r % kOct) + r / kOct;
            }
            ((T *)p.out)[at * D + ch] = sum == 0.f ? (T)0.f : (T)(y[i] * inv);
        }
        if (p.lse && j == 0 && (Few ? lane < 16 : lane < 32)) p.lse[at] = (top + __builtin_amdgcn_logf(sum) - kUnit) * 0.693147180559945f;
    };
    constexpr int kFewPieces = 16;
    if (parts <= kFewPieces) {
#pragma unroll 1
        for (int n = from + wave; n < to; n += kWaves) {
            const int group = n / kBlocks, j = n - group * kBlocks;  // of rows, and the block
            const float4_t *const ml = pieces + (group * (kBlocks + 1) + kBlocks) * 64, *const o = pieces + (group * (kBlocks + 1) + j) * 64;
            const Joined a = join(ml, o, 0, 1);
            write(group, j, a.top, a.sum, a.y);
        }
        return;
    }
#pragma unroll 1
    for (int n = from; n < to; ++n) {
        const int group = n / kBlocks, j = n - group * kBlocks;
        const float4_t *const ml = pieces + (group * (kBlocks + 1) + kBlocks) * 64, *const o = pieces + (group * (kBlocks + 1) + j) * 64;
        const Joined a = join(ml, o, wave, kWaves);
        __syncthreads();  // of the last block's readers
        lds_top[wave][lane] = a.top;
        lds_sum[wave][lane] = a.sum;
        lds_o[wave][lane] = a.y;
        __syncthreads();
        if (wave != n % kWaves) continue;
        float top = -INFINITY, sum = 0.f;
        float4_t y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds_top[w][lane]);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(lds_top[w][lane] - ref);
            sum += lds_sum[w][lane] * f;
            y += lds_o[w][lane] * f;
        }
        write(group, j, top, sum, y);
    }
}

// Rows of a sequence and kv head (the mean) up to which the kernel for few takes them, and up to which weights are in two parts.
constexpr int few_rows(int head_dim, bool eight) { return head_dim == 128 && !eight ? 16 : 64; }
template <int D, bool Eight>
constexpr int kFewRows = few_rows(D, Eight);
constexpr int kTwoRows = 64;

template <typename T, int D, bool Eight>
hipError_t launch_one(const PromptProblem &p, const PromptPlan &plan, hipStream_t stream)
{
    PromptProblem q = p;
    q.target = plan.target;
    q.groups = plan.groups;
    q.records = (char *)p.partials + (size_t)plan.groups * plan.slot_floats * sizeof(float);  // behind the pieces
    const void *kernel, *join;
    if (!plan.few && !plan.two) {
        kernel = (const void *)&prompt_kernel<T, D, Eight, false>;
        join = (const void *)&prompt_join_kernel<T, D, 1, false, Eight, false>;
    } else if (plan.rows == 16) {
        kernel = (const void *)&prompt_few_kernel<T, D, 1, Eight>;
        join = (const void *)&prompt_join_kernel<T, D, 1, true, Eight, true>;
    } else if constexpr (kFewRows<D, Eight> > 16) {
        kernel = (const void *)&prompt_few_kernel<T, D, 2, Eight>;
        join = (const void *)&prompt_join_kernel<T, D, 2, true, Eight, true>;
    } else {
        kernel = (const void *)&prompt_kernel<T, D, Eight, true>;
        join = (const void *)&prompt_join_kernel<T, D, 1, false, Eight, true>;
    }
    const int64_t most = ((int64_t)1 << 24) / p.kv_heads * p.kv_heads - p.kv_heads;
    for (int64_t base = 0; base < plan.groups; base += most) {  // a launch takes less than 2^32 threads
        q.base = (int)base;
        void *args[] = {&q};
        const uint32_t n = (uint32_t)(plan.groups - base < most ? plan.groups - base : most);
        hipError_t e = hipLaunchKernel(kernel, dim3(n), dim3(64 * kWaves), args, 0, stream);
        if (e == hipSuccess && plan.target) e = hipLaunchKernel(join, dim3(n), dim3(64 * kWaves), args, 0, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t launch_typed(const PromptProblem &p, const PromptPlan &plan, int head_dim, hipStream_t stream)
{
    switch (head_dim) {
    case 64: return p.scales ? launch_one<T, 64, true>(p, plan, stream) : launch_one<T, 64, false>(p, plan, stream);
    case 96: return p.scales ? launch_one<T, 96, true>(p, plan, stream) : launch_one<T, 96, false>(p, plan, stream);
    case 128: return p.scales ? launch_one<T, 128, true>(p, plan, stream) : launch_one<T, 128, false>(p, plan, stream);
    case 256: return p.scales ? launch_one<T, 256, true>(p, plan, stream) : launch_one<T, 256, false>(p, plan, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

PromptPlan plan_prompt(int64_t tokens, int64_t B, int64_t heads, int64_t kv_heads, int head_dim, bool eight, int64_t positions, int cus)
{
    PromptPlan x;
    const int64_t rows = tokens * (heads / kv_heads);  // of one kv head
    const int64_t sequences = B < tokens ? B : tokens;
    // Few rows: as long as registers hold what a wave needs.  16 sequences of 1000 to 8000 tokens, 64 rows of new ones for each of 8
    // kv heads (4 of 256 channels): 41 us by the kernel for few rows, 50 by the other one (64 channels), 48 and 60 (96), 58 and 73 (128, 8 bits), 78 and
    // 98 (256); 96 rows: 52 and 45, 69 and 53, 88 and 66, 101 and 96.  Of 32 sequences of 300 to 8000, whose tiles of 64 rows are as many as run
    // at once here and not there, 57 and 66, 101 and 77, 126 and 96, 194 and 142.  In 16 bits two columns of 128 channels do not fit: 32 sequences, 32
    // rows: 163 and 119 (weights rounded once).
    x.few = rows <= few_rows(head_dim, eight) * sequences;
    x.two = rows <= kTwoRows * sequences;
    x.rows = x.few ? (rows <= 16 * sequences ? 16 : 32) : 32 * kWaves;
    // work-groups that run at once: by the registers, those of many rows by the LDS too
    int per_cu = head_dim == 256 ? 1 : 2;
    if (x.few && head_dim == 64) per_cu = x.rows == 16 ? 4 : 3;
    if (x.few && x.rows == 16 && (head_dim == 96 || (head_dim == 128 && eight))) per_cu = 3;
    const int64_t target = (cus < kKvMaxCus ? cus : kKvMaxCus) * per_cu, least = rows / x.rows * kv_heads, most = (rows / x.rows + sequences) * kv_heads;  // tiles
    const int64_t steps = positions >> 4 >> (x.few ? Few::kShift : Many::kShift);
    x.target = least < target && most < 2 * target && steps >= 2 * (x.few ? Few::kLeast : Many::kLeast) ? (int)target : 0;
    // a tile's last part is not a whole one; and the steps are added up in floats
    x.groups = most + (x.target ? x.target + 2 * kv_heads : 0);
    x.slot_floats = x.few ? 64 * 4 * (x.rows / 16) * (head_dim / 16 + 1) : 64 * kWaves * 4 * (head_dim / 32 * 4 + 1);
    return x;
}

size_t prompt_workspace(const PromptPlan &x)
{
    return x.target ? (size_t)x.groups * (sizeof(Record) + (size_t)x.slot_floats * sizeof(float)) : 0;
}

hipError_t launch_prompt(const PromptProblem &p, const PromptPlan &plan, int head_dim, marlin_dtype_t dtype, hipStream_t stream)
{
    return dtype == MARLIN_BF16 ? launch_typed<__bf16>(p, plan, head_dim, stream) : launch_typed<_Float16>(p, plan, head_dim, stream);
}

}  // namespace marlin
