// New tokens into a paged key-value cache of e4m3 codes: queries and keys rotated by
// their positions, keys and values divided by a power of two that their block of 16
// slots and kv head shares, and rounded to 8 bits.
//
//   s = the least 2^e, -40 <= e <= 40, with max |x| <= 448 * 2^e over the block's new tokens; no less than the block's
//       scale so far where it holds earlier ones, whose codes are rounded anew if it grew
//   code = e4m3(x / s)
//
// Powers of two, as a floating-point code loses nothing by them: an element keeps its four bits of
// significand whatever the block's scale is, until it is 2^-14 of the block's largest; and an older code that is divided by
// 2^n once more keeps its bits too.  Keys go to 8 bits from the fp32 of their rotation, each
// operation of which is rounded on its own: a code is then a function of the inputs however the compiler
// would contract the sums.
//
// A head of a token is D / 16 threads as in append.hip.  One token per sequence: the threads find the maximum among
// themselves.  Prompts: a wave takes a block of 16 slots of one head at a time, holds it in
// registers (D / 4 values a lane), finds its maximum across the lanes and writes the codes, so a key is read once.
//
// Bound by memory: 24 prompts of up to 4096 tokens, 64 heads over 8 of 128 (571 MB read and written) 112 to 120 us, 4.8 to 5.1 TB/s, where a
// copy of 2 GiB takes 4.9.  One token of 32 heads over 8: 2.8 us, a launch and the latency of three loads.
#include <hip/hip_runtime.h>

#include "append.h"
#include "kv.h"

namespace marlin {
namespace {

using namespace dev;

// Threads of a head: D / 16, in a power of two of lanes.
template <int D>
constexpr int kLanes = D == 96 ? 8 : D / 16;

struct Codes {
    uint32_t w[4];  // of two pieces
};

__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < INFINITY; }

// x / s as e4m3, two: at most 448 in magnitude, what is not finite as NaN.
__device__ __forceinline__ float in_range(float x, float inv)
{
    return finite(x) ? __builtin_amdgcn_fmed3f(x * inv, -448.f, 448.f) : __builtin_nanf("");
}

__device__ __forceinline__ Codes encode(const float (&x)[16], float inv)
{
    Codes c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(in_range(x[4 * i], inv), in_range(x[4 * i + 1], inv), 0, false);
        c.w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(in_range(x[4 * i + 2], inv), in_range(x[4 * i + 3], inv), w, true);
    }
    return c;
}

__device__ __forceinline__ Codes rescaled(const Codes &c, float ratio)
{
    typedef float float2_t __attribute__((ext_vector_type(2)));
    Codes y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(c.w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c.w[i], true);
        uint32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * ratio, a[1] * ratio, 0, false);
        y.w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(b[0] * ratio, b[1] * ratio, w, true);
    }
    return y;
}

__device__ __forceinline__ Codes load_codes(const uint8_t *row, Where at)
{
    Codes c;
    __builtin_memcpy(c.w, __builtin_assume_aligned(row + at.first, 8), 8);
    __builtin_memcpy(c.w + 2, __builtin_assume_aligned(row + at.second, 8), 8);
    return c;
}

__device__ __forceinline__ void store_codes(uint8_t *row, Where at, const Codes &c)
{
    __builtin_memcpy(__builtin_assume_aligned(row + at.first, 8), c.w, 8);
    __builtin_memcpy(__builtin_assume_aligned(row + at.second, 8), c.w + 2, 8);
}

// The least power of two, 2^-40 .. 2^40, with a <= 448 times it (448 = 1.75 * 2^8): the exponent of a / 256, and one more past 1.75.
__device__ __forceinline__ float scale_of(float a)
{
    int e = (int)((__builtin_bit_cast(uint32_t, a) + 0x1FFFFFu) >> 23) - 127 - 8;
    e = e < -40 ? -40 : e > 40 ? 40 : e;
    return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
}

__device__ __forceinline__ bool is_scale(float s) { return s >= kLeastScale && s <= kMostScale; }

template <typename T>
__device__ __forceinline__ void widen(const Pieces &x, float (&y)[16])
{
    typedef T vec16 __attribute__((ext_vector_type(16)));
    const vec16 e = __builtin_bit_cast(vec16, x);
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = (float)e[i];
}

// The pieces' sixteen channels in fp32, rotated, each operation rounded.
template <typename T>
__device__ __forceinline__ void rotate_exactly(const AppendProblem &p, const Pieces &x, const Angles &a, Where at, float (&y)[16])
{
#pragma clang fp contract(off)
    widen<T>(x, y);
    if (p.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if ((i < 4 ? at.first : at.second) >= p.rot) continue;
            const float c = a.c[i >> 2][i & 3], s = a.s[i >> 2][i & 3], u = y[2 * i], v = y[2 * i + 1];
            const float uc = u * c, vs = v * s, vc = v * c, us = u * s;
            y[2 * i] = uc - vs;
            y[2 * i + 1] = vc + us;
        }
    } else if (at.second < p.rot) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = a.c[i >> 2][i & 3], s = a.s[i >> 2][i & 3], u = y[i], v = y[i + 8];
            const float uc = u * c, vs = v * s, vc = v * c, us = u * s;
            y[i] = uc - vs;
            y[i + 8] = vc + us;
        }
    }
}

__device__ __forceinline__ float largest(const float (&x)[16])
{
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) a = fmaxf(a, finite(x[i]) ? __builtin_fabsf(x[i]) : 0.f);
    return a;
}

template <int N>
__device__ __forceinline__ float max_over_lanes(float a)
{
#pragma unroll
    for (int d = 1; d < N; d <<= 1) a = fmaxf(a, __shfl_xor(a, d));
    return a;
}

// Where a head's scale of a block of slots lies: `slot` as slot_of gives it (of kv head 0), which: 0 keys, 1 values.
__device__ __forceinline__ float *scale_at(const Append8Problem &p, int64_t slot, int head, int which)
{
    const int64_t page_head = (slot >> p.page_shift) + head;
    const int in_page = (int)(slot & ((1 << p.page_shift) - 1)), per_shift = p.page_shift - 4;
    return p.scales + ((page_head * 2 + which) << per_shift) + (in_page >> 4);
}

// ---- one token per sequence ----
template <typename T, int D>
__global__ void __launch_bounds__(256) append8_token_kernel(const Append8Problem p)
{
    constexpr int kPairs = D / 16, kHeads = 256 / kLanes<D>;
    const int pair = threadIdx.x % kLanes<D>, slabs = (p.heads + 2 * p.kv_heads + kHeads - 1) / kHeads;
    const int b = blockIdx.x / slabs, h = blockIdx.x % slabs * kHeads + threadIdx.x / kLanes<D>;
    if (h >= p.heads + 2 * p.kv_heads) return;
    const bool mine = pair < kPairs;  // of three quarters of the lanes where D is 96; the others go along for the maximum
    const int pos = clamped(p.lengths[b]) - 1;
    const int64_t slot = slot_of(p, b, pos);
    const Where at = mine ? where(p, D, pair) : Where{0, 8};
    if (h < p.heads) {
        if (!mine) return;
        Pieces x{};
        if (slot >= 0)
            x = rotate<T>(p, load_pieces((const T *)p.q + b * p.q_row + h * p.q_head, at), load_angles(p, at, pos), at);
        store_pieces((T *)p.q_out + ((int64_t)b * p.heads + h) * D, at, x);
        return;
    }
    if (slot < 0) return;
    const int which = h >= p.heads + p.kv_heads, kh = h - p.heads - which * p.kv_heads;
    float *const scale = scale_at(p, slot, kh, which);
    const int older = (int)slot & (kBlockSlots - 1);
    const float was = older ? *scale : 0.f;
    float x[16];
    if (which)
        widen<T>(load_pieces((const T *)p.v + b * p.v_row + kh * p.v_head, at), x);
    else
        rotate_exactly<T>(p, load_pieces((const T *)p.k + b * p.k_row + kh * p.k_head, at), load_angles(p, at, pos), at, x);
    float s = scale_of(max_over_lanes<kLanes<D>>(mine ? largest(x) : 0.f));
    const bool held = is_scale(was);  // by earlier tokens
    if (held && was > s) s = was;
    if (!mine) return;
    uint8_t *const to = (uint8_t *)(which ? p.v_cache : p.k_cache) + (slot + ((int64_t)kh << p.page_shift)) * D;
    if (held && s > was) {
        const float ratio = was / s;
        for (int i = 1; i <= older; ++i) store_codes(to - i * D, at, rescaled(load_codes(to - i * D, at), ratio));
    }
    store_codes(to, at, encode(x, 1.f / s));
    if (pair == 0 && s != was) *scale = s;
}

// ---- any number of tokens per sequence ----
// A work-group takes the new tokens of one page of one sequence and four heads of q, of k or of v, as in append.hip; a wave
// takes heads of k and v by itself, block after block.
constexpr int kSlab = 4;

template <typename T, int D>
__global__ void __launch_bounds__(256, 3) append8_prompt_kernel(const Append8Problem p, bool once, int page_base)
{
    constexpr int kPairs = D / 16;
    constexpr int kTokens = 64 / kLanes<D>;               // of a wave at a time
    constexpr int kPasses = kBlockSlots / kTokens;        // over a block
    __shared__ int lds_chunks[kKvMaxBatch / 64];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int pair = lane % kLanes<D>, slot = lane / kLanes<D>;
    const bool mine = pair < kPairs;

    const int q_slabs = (p.heads + kSlab - 1) / kSlab, kv_slabs = (p.kv_heads + kSlab - 1) / kSlab;
    const int in_launch = blockIdx.x / (q_slabs + 2 * kv_slabs), y = blockIdx.x - in_launch * (q_slabs + 2 * kv_slabs);
    const PageTokens part = find_page<4>(p, page_base + in_launch, lane, wave, lds_chunks);
    if (part.b < 0) return;

    const Where at = mine ? where(p, D, pair) : Where{0, 8};
    if (y < q_slabs) {
        const int h0 = y * kSlab, nh = p.heads - h0 < kSlab ? p.heads - h0 : kSlab;
        if (!mine) return;
        for (int pos = part.lo + wave * kTokens + slot; pos < part.hi; pos += 4 * kTokens) {
            const int64_t t = part.from + (pos - part.start);
            T *const out = (T *)p.q_out + (t * p.heads + h0) * D;
            if (slot_of(p, part.b, pos) < 0) {
                for (int j = 0; j < nh; ++j) store_pieces(out + j * D, at, Pieces{});
                continue;
            }
            Pieces x[kSlab];
#pragma unroll
            for (int j = 0; j < kSlab; ++j)
                if (j < nh) x[j] = load_new((const T *)p.q + t * p.q_row + (h0 + j) * p.q_head, at, once);
            const Angles a = load_angles(p, at, pos);
#pragma unroll
            for (int j = 0; j < kSlab; ++j)
                if (j < nh) store_pieces(out + j * D, at, rotate<T>(p, x[j], a, at));
        }
        return;
    }
    const int which = y >= q_slabs + kv_slabs, h = (y - q_slabs - which * kv_slabs) * kSlab + wave;
    if (h >= p.kv_heads) return;
    const T *const src = (const T *)(which ? p.v : p.k) + h * (which ? p.v_head : p.k_head);
    const int64_t row = which ? p.v_row : p.k_row;
    for (int block = part.lo & ~(kBlockSlots - 1); block < part.hi; block += kBlockSlots) {
        // positions first .. last - 1 are new, from the block's first to first - 1 earlier ones of the sequence
        int first = part.lo > block ? part.lo : block, last = part.hi < block + kBlockSlots ? part.hi : block + kBlockSlots;
        if (first < 0) first = 0;
        // positions past the table or the angles are not appended
        const int64_t limit = (int64_t)p.width << p.page_shift;
        if (last > limit) last = (int)limit;
        if (p.rot > 0 && last > p.positions) last = p.positions;
        if (first >= last) continue;
        const int64_t to0 = slot_of(p, part.b, first);
        if (to0 < 0) continue;
        const int64_t base = to0 - (first - block);  // the block's first slot
        float *const scale = scale_at(p, base, h, which);
        const float was = first > block ? *scale : 0.f;
        uint8_t *const cache = (uint8_t *)(which ? p.v_cache : p.k_cache) + (base + ((int64_t)h << p.page_shift)) * D;
        Pieces raw[kPasses];
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int pos = block + i * kTokens + slot;
            raw[i] = pos >= first && pos < last && mine ? load_new(src + (int64_t)(part.from + (pos - part.start)) * row, at, once) : Pieces{};
        }
        float x[kPasses][16], a = 0.f;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int pos = block + i * kTokens + slot;
            if (which)
                widen<T>(raw[i], x[i]);
            else
                rotate_exactly<T>(p, raw[i], pos >= first && pos < last ? load_angles(p, at, pos) : Angles{}, at, x[i]);
            a = fmaxf(a, largest(x[i]));
        }
        float s = scale_of(max_over_lanes<64>(a));
        const bool held = is_scale(was);
        if (held && was > s) s = was;
        const float inv = 1.f / s, ratio = was / s;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int pos = block + i * kTokens + slot;
            uint8_t *const to = cache + (i * kTokens + slot) * D;
            if (!mine || pos >= last) continue;
            if (pos >= first)
                store_codes(to, at, encode(x[i], inv));
            else if (held && s > was)
                store_codes(to, at, rescaled(load_codes(to, at), ratio));
        }
        if (lane == 0) *scale = s;
    }
}

template <typename T, int D>
hipError_t launch_one(const Append8Problem &p, hipStream_t stream)
{
    Append8Problem q = p;
    if (!p.starts) {
        constexpr int kHeads = 256 / kLanes<D>;
        const int slabs = (p.heads + 2 * p.kv_heads + kHeads - 1) / kHeads;
        void *args[] = {&q};
        return hipLaunchKernel((const void *)&append8_token_kernel<T, D>, dim3((uint32_t)p.B * slabs), dim3(256), args, 0, stream);
    }
    // a sequence of n tokens touches at most n / page size + 2 pages
    const int pages = (p.tokens >> p.page_shift) + 2 * (p.B < p.tokens ? p.B : p.tokens);
    const int slabs = (p.heads + kSlab - 1) / kSlab + 2 * ((p.kv_heads + kSlab - 1) / kSlab);
    // Rows read once, past the caches, where they would fill those and pieces fill whole lines of 128 bytes.  64, 96, 128, 160, 256 and 512 MB
    // of rows, 64 + 16 heads of 128, so: 33.6, 45.1, 56.0, 66.2, 101 and 206 us, through the caches 27.6, 44.6, 56.1, 73, 111 and 209; 16 + 4 heads
    // of 256: 37.8, 51.1, 63.2, 72.2, 114 and 230, and 32.0, 51.2, 64.7, 77, 125 and 234.  Heads of 64 and 96 gain nothing at any size
    // (160 MB of 40 + 80 heads of 64: 96 and 93.5, 512 MB 298 and 289; 32 + 16 heads of 96: 89.1 and 87.9, 273 and 265).
    bool once = D % 128 == 0 && (int64_t)p.tokens * (p.heads + 2 * p.kv_heads) * D * 2 > ((int64_t)128 << 20);
    const int most = (1 << 24) / slabs - 1;  // pages of a launch, which takes less than 2^32 threads
    for (int base = 0; base < pages; base += most) {
        void *args[] = {&q, &once, &base};
        const uint32_t n = pages - base < most ? pages - base : most;
        const hipError_t e = hipLaunchKernel((const void *)&append8_prompt_kernel<T, D>, dim3(n * slabs), dim3(256), args, 0, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t launch_typed(const Append8Problem &p, int head_dim, hipStream_t stream)
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

hipError_t launch_append8(const Append8Problem &p, int head_dim, marlin_dtype_t dtype, hipStream_t stream)
{
    return dtype == MARLIN_BF16 ? launch_typed<__bf16>(p, head_dim, stream) : launch_typed<_Float16>(p, head_dim, stream);
}

}  // namespace marlin
