// Attention of one new token per sequence over a paged key-value cache.
//
//   o_h = sum_j p_hj v_j,  p_hj = exp(scale q_h . k_j) / sum_i exp(scale q_h . k_i)
//
// One row of work is a (sequence, kv head, tile of up to 16 query heads that
// share it).  A wave takes a step of 32 keys of a row at a time (16 of wide heads), and
// both products are MFMAs whose columns are the 16 heads, so nothing passes
// between lanes but the maximum:
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
// The work is split evenly however ragged the lengths are: the rows'
// steps are numbered through, every work-group (one a compute unit; where a kv head has
// more than 16 query heads, one a range and tile) takes an equal range of them, found from the lengths on the device, and its eight
// waves share it.  Rows that lie within one wave's share go from its registers
// to the output.  Pieces of rows cut between the waves are joined in LDS; what a
// work-group has of rows cut at its borders it leaves in the workspace, and whoever
// arrives last there joins them, in order.
//
// Bound by memory: a step's 16 KB (d = 128) take a compute unit 0.6 us of its
// share of the bandwidth and 0.1 us of MFMA and vector work.  64 sequences of
// 32768 tokens, 64 heads over 8 (8.6 GB): 1.25 ms, 6.9 TB/s, where a kernel that
// only reads reaches 7.1; one of 131071 tokens: 90 us, 6.0.  Short
// calls are latency: 2 us to the first load of keys, a round trip a step, 4 to
// 6 us where rows are cut between work-groups (77 tokens of 32 heads: 5.4 us,
// one sequence of 8000 tokens over 8 kv heads, 33 MB: 13.6).  Four waves a work-group,
// two work-groups a compute unit: 96 us for the 131071 tokens; eight and two: 99.5.
//
// A cache of e4m3 codes is read as it is: codes become the queries' type in registers, exactly, and scales, one for 16 slots, are a factor of the
// tile's scores and a summand in the exponent of its weights.  The 64 sequences, 4.3 GB in 8 bits: 632 us, 6.8 TB/s;
// 16 of up to 4001 tokens, 32 heads over 8 (57 MB): 17.9, in 16 bits 24.8.  Through a window a row's steps are those of the sinks and of
// the window: 32 sequences of up to 60001 tokens, 64 heads over 8, the last 4096 and 4 sinks seen (321 MB): 59 us, 5.4 TB/s.
#include <hip/hip_runtime.h>

#include "device.h"
#include "kv.h"
#include "kv_device.h"

namespace marlin {
namespace {

using namespace dev;

// Constants of the split, in 16-key tiles.
// A work-group border does not cut a row closer to its ends than min_cut
// (it moves to the end): a cut costs a round trip through the workspace.
// min_cut is a quarter of a range, so that no range grows much, between these: with 6
// throughout, 200 sequences of 1 .. 400 tokens, 32 heads over 8, take 21.4 us and not 19.3, with 16
// throughout, one of 2000 takes 12.2 and not 9.6.
constexpr int kMinCut = 6, kMaxCut = 16;
// What a row costs beyond its steps (queries, output).
constexpr int kRowTiles = 2;
// What a work-group gets at least where there is little.
constexpr int kMinTiles = 8;
// Floats of all contributors to a row from which on they are joined in teams.
constexpr int kTeamFloats = 80 << 10;

__device__ __forceinline__ int cap_tokens(const AttendProblem &p, int n)
{
    const int cap = p.width << p.page_shift;
    return n < 0 ? 0 : n < cap ? n : cap;
}

// What a row's token sees through a window: positions below `sinks` and from `low` to before `end`, in steps of 2^shift keys that
// leave out `skip` of them after the first `sink_steps`.
struct Seen {
    int end, low, sinks, sink_steps, skip, steps;
};
__device__ __forceinline__ Seen seen_of(const AttendProblem &p, int tokens, int shift)
{
    Seen x;
    const int cap = p.width << p.page_shift, up = (1 << shift) - 1;
    x.end = tokens < cap ? tokens : cap;
    x.low = tokens > p.window ? tokens - p.window : 0;
    x.sinks = p.sinks < x.low ? p.sinks : x.low;
    const int all = (x.end + up) >> shift, first = x.low >> shift;
    x.sink_steps = (x.sinks + up) >> shift;
    if (x.sink_steps > all) x.sink_steps = all;
    x.skip = (first < all ? first : all) - x.sink_steps;
    if (x.skip < 0) x.skip = 0;
    x.steps = all - x.skip;
    return x;
}

// Where a range begins or ends: a step of a row.
struct Place {
    int b, row;  // sequence, and its row: kv head
    int step;    // of the row
    int before;  // steps of all rows before it
    int steps;   // the row's (where step > 0)
    int tokens;  // the sequence's (-1: still to be read)
};

// A step: its row, and the table's entries for its 16-key tiles.
template <int KT>
struct Step {
    int b, row, tokens, s;
    int e[KT];
};

// KT: 16-key tiles of a step; Eight: the cache holds e4m3 codes; Window: of a row p.window tokens and the first p.sinks are seen
//
// An 8-bit cache's codes become elements of T in the registers, exactly, and never meet their scales there.  A tile's keys share
// one, which joins the scores' factor, and its values' scale s is a part of the weights: p' = exp2(score + log2 s - m'), where m' is
// the maximum of score + log2 s, is what the second product takes, and the sum of the softmax takes p' / s.  With scales from
// 2^-40 to 2^40 nothing of that sum is lost that fp32 would keep: a weight below 2^-126 in p' is below 2^-86 in the sum, whose
// largest term is 2^-40 at the least.  Of the second product's float16 parts those of a p' below 2^-40 of the largest are lost, which
// need not be a small weight: beside a block of values whose scale is 2^40 times larger it is the largest one.  What is lost is
// that part of the row's largest values, but in a channel where those are zero it may be all there is.
template <typename T, int D, int NW, int KT, bool Eight, bool Window>
__global__ void __launch_bounds__(64 * NW) paged_attention_kernel(const AttendProblem p)
{
    typedef Elem<T> E;
    typedef typename E::vec8 vec8;
    typedef T weights_t __attribute__((ext_vector_type(4 * KT)));
    typedef Step<KT> Step;
    constexpr int kQ = D / 32;                // 16-byte pieces of a key's row per lane
    constexpr int kHalves = D > 128 && !Eight ? 2 : 1;  // pieces of a value's row per lane
    constexpr int kCh = D / 16 / kHalves;     // channels in each
    constexpr int kDw = kCh / 2;              // dwords of output in each
    // Dwords of a lane's piece of a row of values, of codes four channels each (96 channels: four of the first 64, two of the others),
    // and of a key's row: with 16-bit elements 16 bytes of every 64; with codes 16 bytes of every 64 too (96 channels: 8 of every 32).
    constexpr int kValueDw = Eight ? (kCh + 3) / 4 : kDw;
    constexpr bool kBy32 = D % 64 != 0;
    constexpr int kKeyDw = Eight ? D / 16 : kQ * 4;
    constexpr int kAcc = D / 16;
    constexpr int kSlotFloats = kHeadTile * D + 2 * kHeadTile;

    // one piece of a row per wave, and that of the row the range ends in
    __shared__ float4_t lds_acc[NW + 1][kAcc][64];
    __shared__ float lds_m[NW + 1][kHeadTile], lds_l[NW + 1][kHeadTile];
    __shared__ int lds_within[NW], lds_flags[3], lds_first[2], lds_last[2];
    __shared__ int lds_chunks[kKvMaxBatch / 64];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int rows = p.kv_heads;  // of a sequence
    constexpr int kStepKeys = kTileKeys * KT, kRowCost = kRowTiles / KT, kMinSteps = kMinTiles / KT;
    constexpr int kStepShift = KT == 2 ? 5 : 4;
    static_assert(kStepKeys == 1 << kStepShift, "");
    // tokens of a sequence as the rows carry them: with a window what lies past the table counts too
    auto tokens_of = [&](int n) {
        if constexpr (Window) return n < 0 ? 0 : n;
        return cap_tokens(p, n);
    };
    // a sequence without keys still has a step, in which its outputs are written
    auto steps_of = [&](int tokens) {
        if constexpr (Window) {
            const int steps = seen_of(p, tokens, kStepShift).steps;
            return steps > 0 ? steps : 1;
        }
        return tokens > 0 ? (tokens + kStepKeys - 1) / kStepKeys : 1;
    };
    // first position of a row's step, and the end of what there is
    auto position_of = [&](int tokens, int s) {
        if constexpr (Window) {
            const Seen x = seen_of(p, tokens, kStepShift);
            return (s < x.sink_steps ? s : s + x.skip) * kStepKeys;
        }
        return s * kStepKeys;
    };
    auto end_of = [&](int tokens) {
        if constexpr (Window) return cap_tokens(p, tokens);
        return tokens;
    };

    // ---- this work-group's range of steps, and this wave's share of it ----
    // Everything until the first loads of keys is latency: no divisions, the lengths of 64 sequences stay in the lanes,
    // and of more only sums of 64 are kept.
    const int chunks = (p.B + 63) / 64;
    int held = -1, length = 0, count = 0, incl = 0;  // chunk in the lanes: tokens, steps, steps up to and with the lane's
    auto hold = [&](int chunk) {
        held = chunk;
        const int b = chunk * 64 + lane;
        length = b < p.B ? tokens_of(p.lengths[b]) : 0;
        count = b < p.B ? steps_of(length) : 0;
        incl = wave_scan(count);
    };
    int total = 0;
    if (chunks == 1) {
        hold(0);
        total = __builtin_amdgcn_readlane(incl, 63);
    } else {
        for (int chunk = wave; chunk < chunks; chunk += NW) {
            hold(chunk);
            if (lane == 63) lds_chunks[chunk] = incl;
        }
        __syncthreads();
        for (int c0 = 0; c0 < chunks; c0 += 64)
            total += __builtin_amdgcn_readlane(wave_scan(c0 + lane < chunks ? lds_chunks[c0 + lane] : 0), 63);
    }
    const int units = (total + kRowCost * p.B) * rows;
    // Range w starts at unit w * units / grid, rounded down, which puts borders between rows of one length; or, where
    // there are few, at w * kMinSteps.
    // A larger group's head tiles read the same keys: the work-groups of a range, one a tile, are neighbours on one XCD, whose L2
    // they share (173 sequences of 4859 tokens, 32 heads over 1: 98 us, spread over the XCDs 131; 16 of 300 .. 30000, 64 over 2: 33.3,
    // 43.5).  Other ranges share nothing, and neighbours on one XCD are no different (64 sequences of 32768 tokens 1249 us, spread
    // 1245; 16 of 500 .. 4001 25.0, 24.9; one of 2000 9.75, 9.8).
    const int tiles = p.head_tiles, grid = tiles == 1 ? gridDim.x : gridDim.x / tiles;
    const int place = tiles == 1 ? blockIdx.x : xcd_local_wg(blockIdx.x, gridDim.x);
    const int wg = tiles == 1 ? place : place / tiles, tile = place - wg * tiles;
    const bool few = units < grid * kMinSteps;
    int per = kMinSteps, extra = 0;
    if (!few) {
        per = (int)__umulhi((uint32_t)units, p.grid_reciprocal);
        extra = units - per * grid;
        if (extra >= grid) {
            ++per;
            extra -= grid;
        }
    }
    if (few && wg * kMinSteps >= units) return;
    const int min_cut = (per / 4 * KT < kMinCut ? kMinCut : per / 4 * KT < kMaxCut ? per / 4 * KT : kMaxCut) / KT;
    auto start_of = [&](int w) {
        // w * extra / grid: exact, as both are below 2^9 and the reciprocal, rounded up, is less than 1 too large
        const int u = w * per + (int)__umulhi((uint32_t)(w * extra), p.grid_reciprocal + 1);
        return u < units ? u : units;
    };
    // smallest w whose range starts at x or later; largest whose starts at x or before
    auto first_at = [&](int x) {
        return few ? (x + kMinSteps - 1) / kMinSteps : (int)(((double)x * grid + (units - 1)) / (double)units);
    };
    auto last_at = [&](int x) {
        return few ? x / kMinSteps : (int)(((double)(x + 1) * grid - 1) / (double)units);
    };
    // the row that holds unit u of the numbering in which a row counts its steps and `cost` more
    auto place_of = [&](int u, int cost) -> Place {
        int before = 0;  // steps of the sequences before the chunk
        if (chunks > 1) {
            int chunk = chunks;
            for (int c0 = 0; c0 < chunks; c0 += 64) {
                const int c = c0 + lane < chunks ? lds_chunks[c0 + lane] : 0, i = wave_scan(c);
                const int last = (c0 + lane + 1) * 64;
                const int ends = c0 + lane < chunks ? (before + i + cost * (last < p.B ? last : p.B)) * rows : 0;
                const uint64_t past = __builtin_amdgcn_ballot_w64(ends > u);
                if (past) {
                    const int at = __builtin_ctzll(past);
                    chunk = c0 + at;
                    before += __builtin_amdgcn_readlane(i, at) - __builtin_amdgcn_readlane(c, at);
                    break;
                }
                before += __builtin_amdgcn_readlane(i, 63);
            }
            if (chunk < chunks && chunk != held) hold(chunk);
        }
        const int b0 = held * 64;
        const int ends = b0 + lane < p.B ? (before + incl + cost * (b0 + lane + 1)) * rows : 0;
        const uint64_t past = __builtin_amdgcn_ballot_w64(ends > u);
        if (u >= units - (kRowCost - cost) * p.B * rows) return {p.B, 0, 0, total * rows, 1, 0};
        const int at = __builtin_ctzll(past);
        const int cb = __builtin_amdgcn_readlane(count, at);
        const int off = u - __builtin_amdgcn_readlane(ends, at) + (cb + cost) * rows;
        // off / (cb + cost): the lanes count the rows that end by then.  The last row's does not, and lanes from there on have none: their
        // products pass 32 bits for 2^30 tokens of wide heads (64 * 2^26 steps), those of the others are units of the numbering.
        const int row = rows == 1 ? 0
                        : rows <= 64 ? __popcll(__builtin_amdgcn_ballot_w64(lane + 1 < rows && (lane + 1) * (cb + cost) <= off))
                                     : (uint32_t)off / (uint32_t)(cb + cost);
        const int step = off - row * (cb + cost) - cost;
        return {b0 + at, row, step < 0 ? 0 : step, u - off - cost * (b0 + at) * rows + row * cb, cb, __builtin_amdgcn_readlane(length, at)};
    };
    auto border = [&](int w) -> Place {
        Place x = place_of(start_of(w), kRowCost);
        if (x.step < min_cut) {
            x.step = 0;
        } else if (x.steps - x.step < min_cut) {
            x.step = 0;
            x.before += x.steps;
            if (++x.row == rows) {
                x.row = 0;
                ++x.b;
                x.tokens = -1;
            }
        }
        return x;
    };
    const Place wg_from = border(wg), wg_to = border(wg + 1);
    const int begin = wg_from.before + wg_from.step, steps = wg_to.before + wg_to.step - begin;
    // Uneven shares: more to the first waves, whose loads are served first (77 tokens of 32 heads: 5.6 us, to the last
    // waves 5.75; 20 sequences, heads of 256: 26.3, 27.7).
    const int share = steps / NW, odd = steps % NW;
    const int mine = share * wave + (wave < odd ? wave : odd);
    int left = share + (wave < odd ? 1 : 0);  // steps of this wave
    Place from = wg_from, to = wg_to;
    if (wg_from.before == wg_to.before) {  // all in one row
        from.step += mine;
        to.step = from.step + left;
    } else {
        if (wave > 0) from = place_of(begin + mine, 0);
        if (wave < NW - 1) to = place_of(begin + mine + left, 0);
    }

    // ---- the steps ----
    // a row's first query head of this work-group's, and how many they are
    auto head0_of = [&](int row) { return row * p.group + tile * kHeadTile; };
    const int nh = p.group - tile * kHeadTile < kHeadTile ? p.group - tile * kHeadTile : kHeadTile;
    auto table_of = [&](const Step &x) {
        return p.table + x.b * p.table_row + x.row * p.table_head;
    };
    // the entries' loads (scalar) are issued a step before they are needed; past the row's tokens nothing is read
    auto entries = [&](Step &x) {
        const int32_t *table = table_of(x);
        const int pos = position_of(x.tokens, x.s), end = end_of(x.tokens);
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            x.e[u] = -1;
            if (pos + kTileKeys * u < end) x.e[u] = scalar_load(table + ((pos + kTileKeys * u) >> p.page_shift));
        }
    };
    auto advance = [&](Step x) -> Step {
        if (x.s + 1 < steps_of(x.tokens)) {
            ++x.s;
        } else {
            x.s = 0;
            if (++x.row == rows) {
                x.row = 0;
                ++x.b;
                x.tokens = tokens_of(scalar_load(p.lengths + x.b));
            }
        }
        entries(x);
        return x;
    };
    vec8 qf[kQ];
    uint32_t kf[KT][kKeyDw] = {};
    uint32_t vr[KT][4][kHalves][kValueDw] = {};
    float key_scale[KT], value_scale[KT];  // of the step whose keys are in the registers; of the other values are under way
    auto load_queries = [&](const Step &x) {
        const T *q = (const T *)p.q + x.b * p.q_row + (head0_of(x.row) + r) * p.q_head + 8 * g;
        const bool have = r < nh;
#pragma unroll
        for (int t = 0; t < kQ; ++t)  // of 16-byte pieces of codes, the halves one after the other
            qf[t] = !have ? vec8{} : *(const vec8 *)(Eight && !kBy32 ? q + 8 * g + 64 * (t >> 1) + 8 * (t & 1) : q + 32 * t);
    };
    // a tile's first element in the caches; an entry that names no page is read as page 0 and masked
    auto tile_at = [&](const Step &x, int u) -> int64_t {
        const int e = x.e[u], kvh = x.row;
        const int slot = (position_of(x.tokens, x.s) + kTileKeys * u) & ((1 << p.page_shift) - 1);
        return ((((int64_t)((uint32_t)e < (uint32_t)p.pages ? e : 0) * p.kv_heads + kvh) << p.page_shift) + slot) * D;
    };
    // Values are read once, whole rows at a time: non-temporal (131071 tokens, 537 MB: 90.2 us, 98.5 through the caches; 16 sequences
    // of up to 4001: 24.9, 27.3).  A load of keys takes 64 bytes of a row, the other half of a line following at once, and goes through
    // the caches: non-temporal, it is within 2 % on large calls, some faster, some slower (128 ragged sequences, 867 MB: 141.0 us, not
    // 143.2; 131071 tokens: 93.5, not 92.6; 64 sequences of 32768: 1315, not 1305), and slower on small ones (16 of up to 4001: 27.1).
    auto load_keys = [&](const Step &x) {
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            if (u > 0 && position_of(x.tokens, x.s) + kTileKeys * u >= end_of(x.tokens)) break;  // masked, whatever the registers hold
            if constexpr (!Eight) {
                const T *k = (const T *)p.k + tile_at(x, u);
#pragma unroll
                for (int t = 0; t < kQ; ++t)
                    __builtin_memcpy(&kf[u][4 * t], __builtin_assume_aligned(k + (r * D + 8 * g) + 32 * t, 16), 16);
            } else {
                const uint8_t *k = (const uint8_t *)p.k + tile_at(x, u) + r * D;
                constexpr int kPiece = kBy32 ? 8 : 16;
#pragma unroll
                for (int t = 0; t < D / (4 * kPiece); ++t)
                    __builtin_memcpy(&kf[u][kPiece / 4 * t], __builtin_assume_aligned(k + kPiece * (g + 4 * t), kPiece), kPiece);
            }
        }
    };
    auto load_values = [&](const Step &x) {
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            if (u > 0 && position_of(x.tokens, x.s) + kTileKeys * u >= end_of(x.tokens)) break;
            if constexpr (!Eight) {
                const T *v = (const T *)p.v + tile_at(x, u);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf)
                        load_dwords_once<kDw>(vr[u][i][hf], v + (4 * g * D + kCh * r) + i * D + 128 * hf);
            } else {
                const uint8_t *v = (const uint8_t *)p.v + tile_at(x, u) + 4 * g * D;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (kBy32) {
                        vr[u][i][0][0] = __builtin_nontemporal_load((const uint32_t *)(v + i * D + 4 * r));
                        vr[u][i][0][1] = __builtin_nontemporal_load((const uint16_t *)(v + i * D + 64 + 2 * r));
                    } else {
                        load_dwords_once<kValueDw>(vr[u][i][0], v + i * D + kCh * r);
                    }
                }
            }
        }
    };
    auto load_scales = [&](const Step &x, float (&of_keys)[KT], float (&of_values)[KT]) {
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            const int e = x.e[u], per_shift = p.page_shift - 4;  // blocks of a page
            const int slot = (position_of(x.tokens, x.s) + kTileKeys * u) & ((1 << p.page_shift) - 1);
            const int64_t head = (int64_t)((uint32_t)e < (uint32_t)p.pages ? e : 0) * p.kv_heads + x.row;
            const float *s = p.scales + ((head * 2) << per_shift) + (slot >> 4);
            of_keys[u] = scalar_load(s);
            of_values[u] = scalar_load(s + (1 << per_shift));
        }
    };
    float4_t acc[kAcc];
    float m, l;
    // slots and counters of this tile's work-group of range w
    auto group_of = [&](int w) { return w * tiles + tile; };
    auto clear = [&] {
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc[j] = float4_t{0.f, 0.f, 0.f, 0.f};
        m = -INFINITY;
        l = 0.f;
    };
    // Joins another piece of the row: its maximum, its sum (each lane that of head r), its accumulators.
    auto join = [&](float m2, float l2, const float4_t(&acc2)[kAcc]) {
        const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
        const float f = __builtin_amdgcn_exp2f(m - ref), f2 = __builtin_amdgcn_exp2f(m2 - ref);
        m = top;
        l = l * f + l2 * f2;
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc[j] = acc[j] * f + acc2[j] * f2;
    };
    auto put_piece = [&](int slot) {
#pragma unroll
        for (int j = 0; j < kAcc; ++j) lds_acc[slot][j][lane] = acc[j];
        if (g == 0) {
            lds_m[slot][r] = m;
            lds_l[slot][r] = l;
        }
    };
    auto join_piece = [&](int slot) {
        float4_t acc2[kAcc];
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc2[j] = lds_acc[slot][j][lane];
        join(lds_m[slot][r], lds_l[slot][r], acc2);
    };
    // The finished row: lane (r, g) holds head r's channels kCh (4g + i) + j.
    auto write_row = [&](int b, int row) {
        if (r >= nh) return;
        const int64_t at = (int64_t)b * p.heads + head0_of(row) + r;
        const float inv = 1.f / (l * E::kWeightUnit);
#pragma unroll
        for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                T y[kCh];
#pragma unroll
                for (int j = 0; j < kCh; ++j) y[j] = l == 0.f ? (T)0.f : (T)(acc[hf * kCh + j][i] * inv);  // no weight: zero, whatever the values
                uint32_t w[kDw];
                __builtin_memcpy(w, y, sizeof(y));
                T *const to = (T *)p.out + at * D;
                if constexpr (Eight && kBy32) {
                    __builtin_memcpy(__builtin_assume_aligned(to + 4 * (4 * g + i), 8), w, 8);
                    __builtin_memcpy(__builtin_assume_aligned(to + 64 + 2 * (4 * g + i), 4), w + 2, 4);
                } else {
                    store_dwords<kDw>(to + 128 * hf + kCh * (4 * g + i), w);
                }
            }
        if (p.lse && g == 0) p.lse[at] = (m + __builtin_amdgcn_logf(l)) * 0.693147180559945f;
    };

    bool begun_before = from.step > 0;  // the row at hand began in another wave
    clear();  // a wave without steps between two that share a row adds nothing to it
    if (left > 0) {
        Step cur{from.b, from.row, from.tokens >= 0 ? from.tokens : tokens_of(scalar_load(p.lengths + from.b)), from.step, {}}, next;
        entries(cur);
        load_queries(cur);
        load_keys(cur);
        load_values(cur);
        if constexpr (Eight) load_scales(cur, key_scale, value_scale);
        if (left > 1) next = advance(cur);
        while (true) {
            float4_t sc[KT];
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                sc[u] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < kQ; ++t) {
                    vec8 x;
                    if constexpr (Eight)
                        x = E::of_codes(kf[u][2 * t], kf[u][2 * t + 1]);
                    else
                        __builtin_memcpy(&x, &kf[u][4 * t], 16);
                    sc[u] = E::mfma(x, qf[t], sc[u]);
                }
            }
            // The next step's keys are under way while this one's scores and values are dealt with,
            // its values while the next scores are.
            const bool row_ends = cur.s + 1 == steps_of(cur.tokens);
            Step ahead;
            float next_key_scale[KT] = {}, next_value_scale[KT] = {};
            issue_order_point();
            if (left > 1) {
                if (row_ends) load_queries(next);
                load_keys(next);
                if constexpr (Eight) load_scales(next, next_key_scale, next_value_scale);
                if (left > 2) ahead = advance(next);
            }
            bool none = (uint32_t)cur.e[0] >= (uint32_t)p.pages || (uint32_t)cur.e[KT - 1] >= (uint32_t)p.pages;
            float add[KT] = {}, times[KT] = {};  // of a tile's scores, of its weights in the sum
            if constexpr (Eight) {
#pragma unroll
                for (int u = 0; u < KT; ++u) {
                    const bool fine = key_scale[u] >= kLeastScale && key_scale[u] <= kMostScale && value_scale[u] >= kLeastScale &&
                                      value_scale[u] <= kMostScale;
                    if (!fine) cur.e[u] = -1;
                    none |= !fine;
                    add[u] = fine ? __builtin_amdgcn_logf(value_scale[u]) : 0.f;
                    times[u] = fine ? __builtin_amdgcn_rcpf(value_scale[u]) : 0.f;
                }
            }
#pragma unroll
            for (int u = 0; u < KT; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (Eight)
                        sc[u][i] = __builtin_fmaf(sc[u][i], p.scale_log2 * key_scale[u], add[u]);
                    else
                        sc[u][i] *= p.scale_log2;
                }
            const int pos = position_of(cur.tokens, cur.s), end = end_of(cur.tokens);
            bool cut = pos + kStepKeys > end || none;
            int low = 0, sinks = 0;
            if constexpr (Window) {
                const Seen x = seen_of(p, cur.tokens, kStepShift);
                low = x.low;
                sinks = x.sinks;
                cut |= pos < low && pos + kStepKeys > sinks;
            }
            if (cut) {
                // Whatever a masked slot holds (an infinity, not a number) stays out of both products.  Selects: the compiler (ROCm 7.2) has
                // dropped assignments to elements of MFMA results in divergent branches, and scores are not far from being those.
#pragma unroll
                for (int u = 0; u < KT; ++u) {
                    const int from_tile = pos + kTileKeys * u;
                    const int valid = (uint32_t)cur.e[u] < (uint32_t)p.pages ? end - from_tile : 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at = 4 * g + i, j = from_tile + at;
                        const bool off = (at >= valid) | (Window & (j < low) & (j >= sinks));
                        sc[u][i] = off ? -INFINITY : sc[u][i];
#pragma unroll
                        for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                            for (int w = 0; w < kValueDw; ++w) vr[u][i][hf][w] = off ? 0 : vr[u][i][hf][w];
                    }
                }
            }
            float top = m;
#pragma unroll
            for (int u = 0; u < KT; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[u][i]);
            top = max_over_groups(top);
            const float ref = top == -INFINITY ? 0.f : top;  // nothing but -inf so far: weights 0
            if (__any(top > m)) {
                const float keep = __builtin_amdgcn_exp2f(m - ref);
                l *= keep;
#pragma unroll
                for (int j = 0; j < kAcc; ++j) acc[j] *= keep;
            }
            m = top;
            float pr[KT][4];
#pragma unroll
            for (int u = 0; u < KT; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) pr[u][i] = __builtin_amdgcn_exp2f(sc[u][i] - ref);
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                const float sum = (pr[u][0] + pr[u][1]) + (pr[u][2] + pr[u][3]);
                l += Eight ? sum * times[u] : sum;
            }
            // The second product takes the weights in the cache's type, as its MFMAs want them, in two parts: rounded down, and what
            // that left out, rounded.  Together they hold 21 bits of a float16 cache's weights and 15 of a bfloat16 one's,
            // float16's times 2^15, so that those far below the maximum are no subnormals (an absolute 2^-40 of it is all that is lost).
            // Both parts of a weight (that is not lost) are above zero, so that an infinite value stays what it is.  (Rounded to
            // nearest, and parted anew where a value is infinite: 77 tokens of 32 heads 5.70 us, this 5.45, weights in one part 5.15.)
            weights_t pf, rest;
#pragma unroll
            for (int e = 0; e < 4 * KT; e += 2) {
                const typename E::Parts x = E::part(pr[e >> 2][e & 3], pr[e >> 2][(e & 3) + 1]);
                pf[e] = x.first[0];
                pf[e + 1] = x.first[1];
                rest[e] = x.rest[0];
                rest[e + 1] = x.rest[1];
            }
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                for (int j = 0; j < kCh; ++j) {
                    uint32_t w[2 * KT];
#pragma unroll
                    for (int e = 0; e < 2 * KT; ++e) {
                        if constexpr (Eight)  // two keys' codes of channels j and j ^ 1 beside each other, of which one pair becomes elements
                            w[e] = E::of_two_codes(__builtin_amdgcn_perm(vr[e >> 1][2 * (e & 1) + 1][hf][j >> 2], vr[e >> 1][2 * (e & 1)][hf][j >> 2],
                                                                         (j & 2) ? 0x07030602u : 0x05010400u), j & 1);
                        else
                            w[e] = __builtin_amdgcn_perm(vr[e >> 1][2 * (e & 1) + 1][hf][j >> 1], vr[e >> 1][2 * (e & 1)][hf][j >> 1],
                                                         (j & 1) ? 0x07060302u : 0x05040100u);
                    }
                    const weights_t x = __builtin_bit_cast(weights_t, w);
                    acc[hf * kCh + j] = E::mfma(x, pf, acc[hf * kCh + j]);
                    acc[hf * kCh + j] = E::mfma(x, rest, acc[hf * kCh + j]);
                }
            issue_order_point();
            if (left > 1) load_values(next);
            if (row_ends || left == 1) l = sum_over_groups(l);
            if (row_ends) {
                if (begun_before)
                    put_piece(wave);
                else
                    write_row(cur.b, cur.row);
                begun_before = false;
                if (left > 1) clear();
            }
            if (--left == 0) break;
            cur = next;
            next = ahead;
            if constexpr (Eight) {
#pragma unroll
                for (int u = 0; u < KT; ++u) {
                    key_scale[u] = next_key_scale[u];
                    value_scale[u] = next_value_scale[u];
                }
            }
        }
    }

    // ---- rows cut between waves ----
    const bool wg_head = wg_from.step > 0, wg_tail = wg_to.step > 0;  // the first row began before, the last goes on after
    const bool one_row = wg_head && wg_from.before == wg_to.before;   // the whole range lies in one row
    const bool open = to.step > 0;             // this wave's last row goes on in the next one; its piece is in the registers
    const bool within = open && begun_before;  // and began in an earlier one: nothing but a piece of it here
    const bool ends_range = open && !within && wg_tail && to.before == wg_to.before;
    if (within) put_piece(wave);
    if (ends_range) put_piece(NW);
    if (lane == 0) lds_within[wave] = within;
    // Contributors to the rows cut at the range's borders (0: the first row, 1: the last): the work-group that holds
    // the row's start, and those whose ranges start within it.  The first wave, which is done early, sees to it.
    if (wave == 0 && (wg_head || wg_tail)) {
        const Place x = lane == 0 ? wg_from : wg_to;
        const int unit = x.before + kRowCost * (x.b * rows + x.row + 1);  // of the row's first step
        const int first = first_at(unit + min_cut) - 1, last = last_at(unit + x.steps - min_cut);
        if (lane < 2) {
            lds_first[lane] = first;
            lds_last[lane] = last;
        }
    }
    __syncthreads();
    if (open && !within && !ends_range) {  // a row that ends in a later wave of this work-group
        bool more = true;
#pragma unroll 1
        for (int w = wave + 1; more; ++w) {
            join_piece(w);
            more = lds_within[w];
        }
        write_row(to.b, to.row);
    }
    if (!wg_head && !wg_tail) return;

    // ---- rows cut between work-groups ----
    // Their pieces (bits of `slots`) are joined by all waves, each some of the channels.
    auto join_slots = [&](uint32_t slots, auto &&put) {
        float mk[NW + 1], lk[NW + 1], top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int k = 0; k <= NW; ++k)
            if (slots >> k & 1) {
                mk[k] = lds_m[k][r];
                lk[k] = lds_l[k][r];
            }
#pragma unroll
        for (int k = 0; k <= NW; ++k)
            if (slots >> k & 1) top = fmaxf(top, mk[k]);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int k = 0; k <= NW; ++k)
            if (slots >> k & 1) {
                mk[k] = __builtin_amdgcn_exp2f(mk[k] - ref);
                sum += lk[k] * mk[k];
            }
#pragma unroll 1
        for (int j = wave; j < kAcc; j += NW) {
            float4_t o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k <= NW; ++k)
                if (slots >> k & 1) o += lds_acc[k][j][lane] * mk[k];
            put(j, o, top, sum);
        }
    };
    const uint32_t all = (1u << NW) - 1;
    const uint32_t inner = (uint32_t)__builtin_amdgcn_ballot_w64(lane < NW && lds_within[lane < NW ? lane : 0]);
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        if (which == 0 ? !wg_head : !wg_tail || one_row) continue;
        // the first row: the waves within it from the first on and the one that ends it; the last: its first piece
        // and the waves after that one
        const uint32_t slots = which == 0 ? (inner == all ? all : ((~inner & (inner + 1)) << 1) - 1)
                                          : (all & ~((2u << (31 - __builtin_clz(~inner & all))) - 1)) | 1u << NW;
        float *const slot = p.partials + ((int64_t)group_of(wg) * 2 + which) * kSlotFloats;
        auto put = [&](int j, float4_t o, float top, float sum) {
            if (r >= nh) return;
            store_partial16(slot, j, lane, o);
            if (j == 0 && g == 0) {
                store_float(slot + kHeadTile * D + r, top);
                store_float(slot + kHeadTile * D + kHeadTile + r, sum);
            }
        };
        // a row through the whole range, without branches: one sequence of 8000 tokens 13.6 us, with them 14.0 (heads of
        // 256: 20 ragged ones 27.7, with them 26.4, though 16 of 30000 157, with them 164)
        if (D <= 128 && slots == all)
            join_slots(all, put);
        else
            join_slots(slots, put);
    }
    // Many contributors are joined in teams (beside each other, the last to arrive joins the team's pieces into its first
    // one's slot, and the last of those the teams'), as one compute unit reads 57 KB a us at most (one sequence of
    // 102932 tokens, 5 heads of 256 over 1: 30.5 us, all by one work-group 54; 60000, 32 heads of 128 over 1: 18.7, 24.7; joins of 9 to
    // 30 contributors, which take this path in one step, cost 0.2 us more for it).
    constexpr int kTeam = 2 * NW;
    auto in_teams = [&](int n) { return n * nh * D > kTeamFloats; };
    wait_vmcnt<0>();
    __syncthreads();
    if (tid < 2) {
        int flag = 0;
        if (tid == 0 ? wg_head : wg_tail && !one_row) {
            const int first = lds_first[tid], n = lds_last[tid] - first + 1;
            const int team = in_teams(n) ? first + (wg - first) / kTeam * kTeam : -1;
            uint32_t *const ctr = p.counters + kCounterStride * group_of(team < 0 ? first : team) + (team < 0 ? 0 : team == first ? 2 : 1);
            const int others = (team < 0 ? n : first + n - team < kTeam ? first + n - team : kTeam) - 1;
            flag = __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)others;
            if (flag) __hip_atomic_store(ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        lds_flags[tid] = flag;
    }
    __syncthreads();
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        if (!__builtin_amdgcn_readfirstlane(lds_flags[which])) continue;
        const int first = __builtin_amdgcn_readfirstlane(lds_first[which]), last = __builtin_amdgcn_readfirstlane(lds_last[which]);
        const __amdgpu_buffer_rsrc_t partials =
            __builtin_amdgcn_make_buffer_rsrc((void *)p.partials, (short)0, 0x7fffffffu, kBufferFlags);
        const int b = which == 0 ? wg_from.b : wg_to.b, row = which == 0 ? wg_from.row : wg_to.row;
        auto write = [&](int j, float4_t o, float top, float sum) {
            if (r >= nh) return;
            const int64_t at = (int64_t)b * p.heads + head0_of(row) + r;
            const float inv = 1.f / (sum * E::kWeightUnit);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int x = 4 * g + i;
                const int ch = Eight && kBy32 ? (j < 4 ? 4 * x + j : 60 + 2 * x + j) : 128 * (j / kCh) + kCh * x + j % kCh;
                ((T *)p.out)[at * D + ch] = sum == 0.f ? (T)0.f : (T)(o[i] * inv);
            }
            if (p.lse && g == 0 && j == 0) p.lse[at] = (top + __builtin_amdgcn_logf(sum)) * 0.693147180559945f;
        };
        // Contributors are joined in order, so that the bits are the same every time.  Of a few, a wave takes its channels at once
        // (16 sequences of up to 4001 tokens: 24.9 us, by LDS as below 26.1; the registers of both do not go together where heads are wide).
        constexpr int kFew = 8;
        if (D <= 128 && last - first < kFew) {
            if (wave < kAcc && r < nh) {
                const int j = wave;
                float mk[kFew], lk[kFew], top = -INFINITY, sum = 0.f;
                float4_t a[kFew], o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < kFew; ++k)
                    if (first + k <= last) {
                        const int slot = (group_of(first + k) * 2 + (k == 0 ? 1 : 0)) * (kSlotFloats * 4);
                        mk[k] = load_slot4(partials, slot, kHeadTile * D * 4 + r * 4);
                        lk[k] = load_slot4(partials, slot, kHeadTile * D * 4 + kHeadTile * 4 + r * 4);
                        a[k] = load_slot16(partials, slot, j * 1024 + lane * 16);
                    }
#pragma unroll
                for (int k = 0; k < kFew; ++k)
                    if (first + k <= last) top = fmaxf(top, mk[k]);
                const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int k = 0; k < kFew; ++k)
                    if (first + k <= last) {
                        const float f = __builtin_amdgcn_exp2f(mk[k] - ref);
                        sum += lk[k] * f;
                        o += a[k] * f;
                    }
                write(j, o, top, sum);
            }
            continue;
        }
        // Of more, a wave takes some of the contributors, then all take the waves'.
        const bool teams = in_teams(last - first + 1);
        const int team = first + (wg - first) / kTeam * kTeam;
#pragma unroll 1
        for (int level = teams ? 0 : 1; level < 2; ++level) {
            const int begin_w = level == 0 ? team : first, step_w = level == 1 && teams ? kTeam : 1;
            const int end_w = level == 0 && team + kTeam - 1 < last ? team + kTeam - 1 : last;
            clear();
            if (r < nh) {
                struct Piece {
                    float m, l;
                    float4_t acc[kAcc];
                };
                auto load_piece = [&](int w, Piece &x) {
                    const int slot = (group_of(w) * 2 + (w == first ? 1 : 0)) * (kSlotFloats * 4);
#pragma unroll
                    for (int j = 0; j < kAcc; ++j) x.acc[j] = load_slot16(partials, slot, j * 1024 + lane * 16);
                    x.m = load_slot4(partials, slot, kHeadTile * D * 4 + r * 4);
                    x.l = load_slot4(partials, slot, kHeadTile * D * 4 + kHeadTile * 4 + r * 4);
                };
                constexpr int kAhead = 2;  // under way together
#pragma unroll 1
                for (int w = begin_w + wave * step_w; w <= end_w; w += kAhead * NW * step_w) {
                    Piece x[kAhead];
#pragma unroll
                    for (int k = 0; k < kAhead; ++k)
                        if (w + k * NW * step_w <= end_w) load_piece(w + k * NW * step_w, x[k]);
#pragma unroll
                    for (int k = 0; k < kAhead; ++k)
                        if (w + k * NW * step_w <= end_w) join(x[k].m, x[k].l, x[k].acc);
                }
            }
            put_piece(wave);
            __syncthreads();
            float *const slot = p.partials + ((int64_t)group_of(team) * 2 + (team == first ? 1 : 0)) * kSlotFloats;
            join_slots(all, [&](int j, float4_t o, float top, float sum) {
                if (level == 1) return write(j, o, top, sum);
                if (r >= nh) return;
                store_partial16(slot, j, lane, o);
                if (j == 0 && g == 0) {
                    store_float(slot + kHeadTile * D + r, top);
                    store_float(slot + kHeadTile * D + kHeadTile + r, sum);
                }
            });
            if (level == 1) break;
            wait_vmcnt<0>();
            __syncthreads();
            if (tid == 0) {
                uint32_t *const ctr = p.counters + kCounterStride * group_of(first);
                const bool done = __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)((last - first) / kTeam);
                if (done) __hip_atomic_store(ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                lds_flags[2] = done;
            }
            __syncthreads();
            if (!__builtin_amdgcn_readfirstlane(lds_flags[2])) break;
        }
        __syncthreads();
    }
}

template <typename T, int D, bool Eight, bool Window>
hipError_t launch_one(const AttendProblem &p, int cus, hipStream_t stream)
{
    const int groups = (cus < kKvMaxCus ? cus : kKvMaxCus) * kAttendGroupsPerCu;
    const int ranges = groups > p.head_tiles ? groups / p.head_tiles : 1;  // at most 64 tiles
    // Wide heads: one tile a step, which keeps the registers and divides short ranges finer (heads of 256, 20 sequences of up
    // to 9001 tokens 26.4 us, two tiles 29.0; 16 of 30000: 164.4, 165.4).  Narrower ones: two, fewer round trips in short
    // ranges (one sequence of 2000, heads of 128: 9.8 us, one tile 10.7).
    constexpr int kTiles = D > 128 ? 1 : 2;
    AttendProblem q = p;
    q.grid_reciprocal = ranges > 1 ? (uint32_t)(((uint64_t)1 << 32) / (uint64_t)ranges) : 0xFFFFFFFFu;
    void *args[] = {&q};
    return hipLaunchKernel((const void *)&paged_attention_kernel<T, D, kAttendWaves, kTiles, Eight, Window>, dim3(ranges * p.head_tiles),
                           dim3(64 * kAttendWaves), args, 0, stream);
}

template <typename T, int D>
hipError_t launch_cache(const AttendProblem &p, int cus, hipStream_t stream)
{
    if (p.scales) return p.window ? launch_one<T, D, true, true>(p, cus, stream) : launch_one<T, D, true, false>(p, cus, stream);
    return p.window ? launch_one<T, D, false, true>(p, cus, stream) : launch_one<T, D, false, false>(p, cus, stream);
}

template <typename T>
hipError_t launch_typed(const AttendProblem &p, int head_dim, int cus, hipStream_t stream)
{
    switch (head_dim) {
    case 64: return launch_cache<T, 64>(p, cus, stream);
    case 96: return launch_cache<T, 96>(p, cus, stream);
    case 128: return launch_cache<T, 128>(p, cus, stream);
    case 256: return launch_cache<T, 256>(p, cus, stream);
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
