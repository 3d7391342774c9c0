// The page tables of a step: pages that ended sequences and windows leave go back to the free ones,
// new tokens get pages from there, and each its slot (marlin_assign_pages).
//
// All of it follows from sums over the sequences in their order: of pages given back, of pages needed, of new
// tokens.  One work-group scans them, 1024 sequences at a time; as both sums only grow, the
// sequences that are served are those before the first whose pages or tokens are too many (and that fit their rows of
// the table), so what lies before a sequence is the smaller of its own sum and the last served one's.
// A sequence's new pages are all among its new tokens' (each has its first slot there), so
// whoever finds a token's slot takes the page from the free ones by the sums, without a loop over pages.
//
// Latency is all there is: a scan is 1.5 us, a token's slot a search among the sequences and two
// dependent loads.  Up to kFusedTokens new tokens the same work-group finds the slots, more are a second launch.
#include <hip/hip_runtime.h>

#include "kv.h"
#include "kv_device.h"

namespace marlin {
namespace {

using namespace dev;

constexpr int kThreads = 1024, kSums = kThreads / 64;
constexpr int kFusedTokens = 2048;

__device__ __forceinline__ uint32_t add_up(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Sums over the work-group's threads up to and with each, on top of `before`, which becomes the sum of all; saturating.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t &before, uint32_t *lds, int lane, int wave)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(x, d);
        if (lane >= d) x = add_up(x, y);
    }
    __syncthreads();  // of the last scan's readers
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    uint32_t mine = before, all = before;
#pragma unroll
    for (int w = 0; w < kSums; ++w) {
        if (w < wave) mine = add_up(mine, lds[w]);
        all = add_up(all, lds[w]);
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

template <bool Fused>
__global__ void __launch_bounds__(kThreads) assign_kernel(const PagesProblem p)
{
    __shared__ uint32_t lds_sums[kSums];
    __shared__ uint32_t lds_served[2][kSums];
    __shared__ int lds_starts[kThreads + 1], lds_before[kThreads], lds_had[kThreads];  // of up to 1024 sequences
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ps = 1 << p.page_shift, cap = p.width << p.page_shift;
    int count = *p.free_count;
    count = count < 0 ? 0 : count < p.pages ? count : p.pages;

    auto length_of = [&](int b) {
        const int n = p.lengths[b];
        return n < 0 ? 0 : n < cap ? n : cap;
    };

    // ---- given back ----
    uint32_t returned = 0;
    for (int b0 = 0; b0 < p.B; b0 += kThreads) {
        const int b = b0 + tid;
        // entries first .. last - 1 are looked at, all of them (an ended sequence's) or from the last down to one that names no page
        int first = 0, last = 0;
        bool ends = false;
        if (b < p.B) {
            const int had = length_of(b);
            ends = p.new_tokens[b] < 0;
            if (ends) {
                last = (had + ps - 1) >> p.page_shift;
            } else if (p.window > 0 && had > p.window) {
                first = (p.sinks + ps - 1) >> p.page_shift;
                last = (had - p.window) >> p.page_shift;
                if (last > first && (uint32_t)p.table[b * p.table_row + last - 1] >= (uint32_t)p.pages) last = 0;
            }
            if (last <= first) last = first = 0;
        }
        // a wave looks at its 64 sequences' entries one after another, 64 entries at a time
        uint32_t mine = 0;
        const uint64_t work = __builtin_amdgcn_ballot_w64(last > first);
        for (uint64_t left = work; left; left &= left - 1) {
            const int of = __builtin_ctzll(left);
            const int f = __builtin_amdgcn_readlane(first, of), l = __builtin_amdgcn_readlane(last, of);
            const bool whole = __builtin_amdgcn_readlane(ends, of);
            const int32_t *const row = p.table + (int64_t)(b0 + wave * 64 + of) * p.table_row;
            uint32_t n = 0;
            for (int at = l; at > f; at -= 64) {
                const int i = at - 1 - lane;
                const uint64_t named = __builtin_amdgcn_ballot_w64(i >= f && (uint32_t)row[i >= f ? i : f] < (uint32_t)p.pages);
                if (whole) {
                    n += __popcll(named);
                } else {
                    const int run = ~named ? __builtin_ctzll(~named) : 64;
                    n += run;
                    if (run < 64) break;
                }
            }
            if (lane == of) mine = n;
        }
        const uint32_t upto = block_scan(mine, returned, lds_sums, lane, wave);
        // written in ascending order: the run below a window's end is its last `mine` entries
        for (uint64_t left = work; left; left &= left - 1) {
            const int of = __builtin_ctzll(left);
            const int l = __builtin_amdgcn_readlane(last, of), n = __builtin_amdgcn_readlane(mine, of);
            const bool whole = __builtin_amdgcn_readlane(ends, of);
            const int f = whole ? __builtin_amdgcn_readlane(first, of) : l - n;
            int32_t *const row = p.table + (int64_t)(b0 + wave * 64 + of) * p.table_row;
            int64_t to = (int64_t)count + (uint32_t)__builtin_amdgcn_readlane(upto, of) - n;
            for (int at = f; at < l; at += 64) {
                const int i = at + lane;
                const int page = i < l ? row[i] : -1;
                const bool named = (uint32_t)page < (uint32_t)p.pages;
                const uint64_t all = __builtin_amdgcn_ballot_w64(named);
                const int64_t at_free = to + __popcll(all & (((uint64_t)1 << lane) - 1));
                if (named) {
                    if (at_free < p.pages) p.free_pages[at_free] = page;
                    row[i] = -1;
                }
                to += __popcll(all);
            }
        }
    }
    const int room = (int)((int64_t)count + returned < p.pages ? count + returned : p.pages);

    // ---- served ----
    uint32_t pages_sum = 0, tokens_sum = 0, pages_served = 0, tokens_served = 0;
    if (tid == 0) p.starts[0] = 0;
    if (Fused && tid == 0) lds_starts[0] = 0;
    for (int b0 = 0; b0 < p.B; b0 += kThreads) {
        const int b = b0 + tid;
        int had = 0, n = 0;
        if (b < p.B) {
            had = length_of(b);
            n = p.new_tokens[b];
        }
        const bool fits = n > 0 && n <= cap - had;
        const uint32_t need = fits ? ((had + n + ps - 1) >> p.page_shift) - ((had + ps - 1) >> p.page_shift) : 0;
        const uint32_t pages = block_scan(need, pages_sum, lds_sums, lane, wave);
        const uint32_t tokens = block_scan(fits ? n : 0, tokens_sum, lds_sums, lane, wave);
        const bool served = fits && pages <= (uint32_t)room && tokens <= (uint32_t)p.tokens;
        // the last served one's sums
        uint32_t a = served ? pages : 0, c = served ? tokens : 0;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const uint32_t a2 = __shfl_xor(a, d), c2 = __shfl_xor(c, d);
            a = a2 > a ? a2 : a;
            c = c2 > c ? c2 : c;
        }
        if (lane == 0) {
            lds_served[0][wave] = a;
            lds_served[1][wave] = c;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSums; ++w) {
            pages_served = lds_served[0][w] > pages_served ? lds_served[0][w] : pages_served;
            tokens_served = lds_served[1][w] > tokens_served ? lds_served[1][w] : tokens_served;
        }
        if (b < p.B) {
            const uint32_t end = tokens < tokens_served ? tokens : tokens_served;
            const uint32_t before = served ? pages - need : 0;
            p.starts[b + 1] = (int)end;
            if (served)
                p.lengths[b] = had + n;
            else if (n < 0)
                p.lengths[b] = 0;
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
    const hipError_t e = hipLaunchKernel(fused ? (const void *)&assign_kernel<true> : (const void *)&assign_kernel<false>, dim3(1),
                                         dim3(kThreads), args, 0, stream);
    if (e != hipSuccess || fused) return e;
    return hipLaunchKernel((const void *)&slots_kernel, dim3((p.tokens + 255) / 256), dim3(256), args, 0, stream);
}

}  // namespace marlin
