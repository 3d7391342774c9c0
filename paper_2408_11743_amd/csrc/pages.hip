// The page tables of a step: pages that ended sequences, windows and tokens taken back leave go back to the free ones,
// new tokens get pages from there, and each its slot (marlin_assign_pages).
//
// All of it follows from sums over the sequences in their order: of pages given back, of pages needed, of new
// tokens.  One work-group scans them, 1024 sequences at a time; as both sums only grow, the
// sequences that are served are those before the first whose pages or tokens are too many (and that fit their rows of
// the table), so what lies before a sequence is the smaller of its own sum and the last served one's.
// A sequence's new pages are all among its new tokens' (each has its first slot there), so
// whoever finds a token's slot takes the page from the free ones by the sums, without a loop over pages.
//
// Latency is all there is: launch, loads, two scans, a token's slot a search among the sequences and two dependent
// loads (128 sequences of one new token behind windows: 7 us).  Up to kFusedTokens new tokens the same work-group finds the slots, more are a second
// launch: 700 tokens of 16 sequences 8.9 us, by two launches 11.6; 2200 9.2 and 11.7; 6400 12.5 and 11.8; 240000 of 512 sequences 265 and 14.5.
#include <hip/hip_runtime.h>

#include "kv.h"
#include "kv_device.h"

namespace marlin {
namespace {

using namespace dev;

constexpr int kThreads = 1024, kSums = kThreads / 64;
constexpr int kFusedTokens = 4096;

// Two sums over the work-group's threads up to and with each, on top of `before`, which becomes the sums of all; saturating.
struct Two {
    uint32_t a, b;
};
__device__ __forceinline__ Two add_up(Two x, Two y) { return {__builtin_elementwise_add_sat(x.a, y.a), __builtin_elementwise_add_sat(x.b, y.b)}; }
__device__ __forceinline__ Two block_scan(Two x, Two &before, Two *lds, int lane, int wave, int waves)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const Two y{(uint32_t)__shfl_up(x.a, d), (uint32_t)__shfl_up(x.b, d)};
        if (lane >= d) x = add_up(x, y);
    }
    __syncthreads();  // of the last scan's readers
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    Two mine = before, all = before;
    for (int w = 0; w < waves; ++w) {
        const Two y = lds[w];
        if (w < wave) mine = add_up(mine, y);
        all = add_up(all, y);
    }
    before = all;
    return add_up(mine, x);
}

// The sequence that new token t is of: the last whose tokens begin at t or before.
template <typename S>
__device__ __forceinline__ int sequence_of(const S *starts, int B, int t)
{
    int lo = 0, hi = B;  // starts[lo] <= t < starts[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= t)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// A token's slot; the first token of a new page writes its entry.  room: free pages, before: taken before the sequence's.
__device__ __forceinline__ int64_t slot_of_token(const PagesProblem &p, int b, int pos, int had, int before, int room)
{
    const int i = pos >> p.page_shift, have = (had + (1 << p.page_shift) - 1) >> p.page_shift;
    int32_t *const entry = p.table + b * p.table_row + i;
    int page;
    if (i < have) {
        page = *entry;
    } else {
        page = p.free_pages[room - 1 - (before + i - have)];
        if (pos == i << p.page_shift) *entry = page;
    }
    return (uint32_t)page >= (uint32_t)p.pages ? -1 : ((int64_t)page << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
}

// Back: tokens are taken back; a variant, as looking for them took 0.3 us of each call.
template <bool Fused, bool Back>
__global__ void __launch_bounds__(kThreads) assign_kernel(const PagesProblem p)
{
    __shared__ Two lds_sums[kSums], lds_served[kSums];
    __shared__ int lds_starts[kThreads + 1], lds_before[kThreads], lds_had[kThreads];  // of up to 1024 sequences
    // sequences whose entries are looked at: thread, first entry, last (with the sign bit: all of them count); what is given back
    __shared__ int lds_works, lds_of[kThreads], lds_first[kThreads], lds_last[kThreads], lds_given[kThreads], lds_upto[kThreads];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ps = 1 << p.page_shift, cap = p.width << p.page_shift;
    int count = *p.free_count;
    count = count < 0 ? 0 : count < p.pages ? count : p.pages;

    auto whole_length_of = [&](int b) {
        const int n = p.lengths[b];
        return n < 0 ? 0 : n < cap ? n : cap;
    };
    // without the tokens that are taken back
    auto length_of = [&](int b) {
        const int n = whole_length_of(b), back = Back ? p.back[b] : 0;
        return back <= 0 ? n : n > back ? n - back : 0;
    };

    // ---- given back ----
    Two returned{0, 0};
    int had0 = 0, new0 = 0;  // of the first 1024 sequences
    for (int pass = Back ? 0 : 1; pass < 2; ++pass) {  // pages without a token left, then those of ended sequences and behind windows
        const bool taken_back = Back && pass == 0;
        for (int b0 = 0; b0 < p.B; b0 += kThreads) {
            const int b = b0 + tid;
            if (tid == 0) lds_works = 0;
            __syncthreads();
            // entries first .. last - 1 are looked at, all of them (an ended sequence's) or from the last down to one that names no page
            int first = 0, last = 0;
            bool ends = false;
            if (b < p.B) {
                const int had = length_of(b), fresh = p.new_tokens[b];
                if (b0 == 0) {
                    had0 = had;
                    new0 = fresh;
                }
                ends = fresh < 0 || taken_back;
                if (taken_back) {
                    first = (had + ps - 1) >> p.page_shift;
                    last = (whole_length_of(b) + ps - 1) >> p.page_shift;
                } else if (ends) {
                    last = (had + ps - 1) >> p.page_shift;
                } else if (p.window > 0 && had > p.window) {
                    first = (p.sinks + ps - 1) >> p.page_shift;
                    last = (had - p.window) >> p.page_shift;
                    if (last > first && (uint32_t)p.table[b * p.table_row + last - 1] >= (uint32_t)p.pages) last = 0;
                }
            }
            lds_given[tid] = 0;
            if (last > first) {
                const int at = atomicAdd(&lds_works, 1);  // in any order
                lds_of[at] = tid;
                lds_first[at] = first;
                lds_last[at] = ends ? last | 1 << 31 : last;
            }
            __syncthreads();
            const int works = lds_works;
            if (works == 0) continue;
            // a sequence is a wave's, 64 entries at a time
            for (int i = wave; i < works; i += kSums) {
                const int of = lds_of[i], f = lds_first[i], l = lds_last[i] & 0x7FFFFFFF;
                const bool whole = lds_last[i] < 0;
                const int32_t *const row = p.table + (int64_t)(b0 + of) * p.table_row;
                int n = 0;
                for (int at = l; at > f; at -= 64) {
                    const int e = at - 1 - lane;
                    const uint64_t named = __builtin_amdgcn_ballot_w64(e >= f && (uint32_t)row[e >= f ? e : f] < (uint32_t)p.pages);
                    if (whole) {
                        n += __popcll(named);
                    } else {
                        const int run = ~named ? __builtin_ctzll(~named) : 64;
                        n += run;
                        if (run < 64) break;
                    }
                }
                if (lane == 0) lds_given[of] = n;
            }
            __syncthreads();
            const Two upto = block_scan({(uint32_t)lds_given[tid], 0}, returned, lds_sums, lane, wave, kSums);
            lds_upto[tid] = (int)upto.a;
            __syncthreads();
            // written in ascending order: the run below a window's end is its last entries
            for (int i = wave; i < works; i += kSums) {
                const int of = lds_of[i], l = lds_last[i] & 0x7FFFFFFF, n = lds_given[of], f = lds_last[i] < 0 ? lds_first[i] : l - n;
                int32_t *const row = p.table + (int64_t)(b0 + of) * p.table_row;
                int64_t to = (int64_t)count + (uint32_t)lds_upto[of] - n;
                for (int at = f; at < l; at += 64) {
                    const int e = at + lane;
                    const int page = e < l ? row[e] : -1;
                    const bool named = (uint32_t)page < (uint32_t)p.pages;
                    const uint64_t all = __builtin_amdgcn_ballot_w64(named);
                    const int64_t at_free = to + __popcll(all & (((uint64_t)1 << lane) - 1));
                    if (named) {
                        if (at_free < p.pages) p.free_pages[at_free] = page;
                        row[e] = -1;
                    }
                    to += __popcll(all);
                }
            }
        }
    }
    const int room = (int)((int64_t)count + returned.a < p.pages ? count + returned.a : p.pages);

    // ---- served ----
    Two sums{0, 0};
    uint32_t pages_served = 0, tokens_served = 0;
    if (tid == 0) p.starts[0] = 0;
    if (Fused && tid == 0) lds_starts[0] = 0;
    for (int b0 = 0; b0 < p.B; b0 += kThreads) {
        const int b = b0 + tid;
        int had = had0, n = new0;
        if (b0 > 0) {
            had = b < p.B ? length_of(b) : 0;
            n = b < p.B ? p.new_tokens[b] : 0;
        }
        const bool fits = n > 0 && n <= cap - had;
        const uint32_t need = fits ? ((had + n + ps - 1) >> p.page_shift) - ((had + ps - 1) >> p.page_shift) : 0;
        const Two upto = block_scan({need, fits ? (uint32_t)n : 0}, sums, lds_sums, lane, wave, kSums);
        const uint32_t pages = upto.a, tokens = upto.b;
        const bool served = fits && pages <= (uint32_t)room && tokens <= (uint32_t)p.tokens;
        // the last served one's sums: of a wave the last lane's that is
        const uint64_t any = __builtin_amdgcn_ballot_w64(served);
        const int at = any ? 63 - __builtin_clzll(any) : 0;
        const Two most{any ? (uint32_t)__builtin_amdgcn_readlane(pages, at) : 0u, any ? (uint32_t)__builtin_amdgcn_readlane(tokens, at) : 0u};
        if (lane == 0) lds_served[wave] = most;
        __syncthreads();
        for (int w = 0; w < kSums; ++w) {
            const Two x = lds_served[w];
            pages_served = x.a > pages_served ? x.a : pages_served;
            tokens_served = x.b > tokens_served ? x.b : tokens_served;
        }
        if (b < p.B) {
            const uint32_t end = tokens < tokens_served ? tokens : tokens_served;
            const uint32_t before = served ? pages - need : 0;
            p.starts[b + 1] = (int)end;
            if (served)
                p.lengths[b] = had + n;
            else if (n < 0)
                p.lengths[b] = 0;
            else if (Back && p.back[b] > 0)
                p.lengths[b] = had;
            if (Fused) {
                if (p.B <= kThreads) {
                    lds_starts[b + 1] = (int)end;
                    lds_before[b] = (int)before;
                    lds_had[b] = had;
                }
            }
            p.before[b] = (int)before;
        }
    }
    if (tid == 0) {
        *p.free_count = room - (int)pages_served;
        p.before[p.B] = room;
    }
    if (!Fused) return;
    __syncthreads();
    for (int t = tid; t < p.tokens; t += kThreads) {
        int64_t slot = -1;
        if (t < (int)tokens_served) {
            if (p.B <= kThreads) {
                const int b = sequence_of(lds_starts, p.B, t);
                slot = slot_of_token(p, b, lds_had[b] + t - lds_starts[b], lds_had[b], lds_before[b], room);
            } else {
                const int b = sequence_of(p.starts, p.B, t), first = p.starts[b];
                const int had = p.lengths[b] - (p.starts[b + 1] - first);
                slot = slot_of_token(p, b, had + t - first, had, p.before[b], room);
            }
        }
        p.slots[t] = slot;
    }
}

__global__ void __launch_bounds__(256) slots_kernel(const PagesProblem p)
{
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= p.tokens) return;
    int64_t slot = -1;
    if (t < p.starts[p.B]) {
        const int b = sequence_of(p.starts, p.B, t), first = p.starts[b];
        const int had = p.lengths[b] - (p.starts[b + 1] - first);
        slot = slot_of_token(p, b, had + t - first, had, p.before[b], p.before[p.B]);
    }
    p.slots[t] = slot;
}

}  // namespace

hipError_t launch_pages(const PagesProblem &p, hipStream_t stream)
{
    PagesProblem q = p;
    void *args[] = {&q};
    const bool fused = p.tokens <= kFusedTokens;
    const void *const kernel = !p.back ? (fused ? (const void *)&assign_kernel<true, false> : (const void *)&assign_kernel<false, false>)
                                       : (fused ? (const void *)&assign_kernel<true, true> : (const void *)&assign_kernel<false, true>);
    const hipError_t e = hipLaunchKernel(kernel, dim3(1), dim3(kThreads), args, 0, stream);
    if (e != hipSuccess || fused) return e;
    return hipLaunchKernel((const void *)&slots_kernel, dim3((p.tokens + 255) / 256), dim3(256), args, 0, stream);
}

}  // namespace marlin
