// Device code that the kernels of the paged cache share (wkv_paged.hip, wkv_flash.hip): matrix instructions by format, rounding
// to 16 bits, and what a sequence, a tile of rows and a part of its keys are.  Each kernel file gets its own copy.
#ifndef WKV_PAGED_DEVICE_H
#define WKV_PAGED_DEVICE_H

#include "wkv_device.h"
#include "wkv_internal.h"

namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

constexpr int ROWS = 16;            // rows of a tile, and of a cell of the workspace

template <class TT> __device__ __forceinline__ f32x4_t mfma(u32x4_t a, u32x4_t b, f32x4_t c)
{
    if constexpr (__is_same(TT, TF16))
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mfma_f32(float a, float b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Two floats to two 16-bit elements, nearest even.
template <class TT> __device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    if constexpr (__is_same(TT, TF16)) {
        const half2_t h = {(_Float16)lo, (_Float16)hi};
        return __builtin_bit_cast(uint32_t, h);
    } else {
        const bf16x2_t h = {(__bf16)lo, (__bf16)hi};
        return __builtin_bit_cast(uint32_t, h);
    }
}
template <class TT> __device__ __forceinline__ void unpack2(uint32_t w, float& lo, float& hi)
{
    if constexpr (__is_same(TT, TF16)) {
        const half2_t h = __builtin_bit_cast(half2_t, w);
        lo = (float)h.x; hi = (float)h.y;
    } else {
        lo = __builtin_bit_cast(float, w << 16); hi = __builtin_bit_cast(float, w & 0xFFFF0000u);
    }
}

// Weights are 2^(logit - reference), the reference being a logit (log2) that none exceeds by more than 8 (fp16: a number that none exceeds by
// more than 15), so sums of 16-bit values up to 2^128 and of fp32 values may leave the range of fp32 although their mean does not.  Such a sum is
// formed anew with every weight times 2^-CAREFUL, which is a larger reference (a sequence has at most 2^24 slots); a reference that is larger from
// the start would cost the exponents of all weights 5 bits.  Where sums of several waves or parts are joined, the common reference is JOINED above
// the largest.
template <class TT> constexpr float CAREFUL = __is_same(TT, TF16) ? 0.f : 32.f;
constexpr float JOINED = 8.f;

// A row's output from its sum of weight . v.  It is a mean of values, so roundings must not take it over the format's largest number.
template <class TT> __device__ __forceinline__ float mean(float sum, float inv)
{
    constexpr float MOST = __is_same(TT, TF16) ? 65504.f : __is_same(TT, TBF16) ? 0x1.FEp127f : 0x1.FFFFFEp127f;
    const float x = sum * inv;
    return __builtin_isinf(sum) ? x : x > MOST ? MOST : x < -MOST ? -MOST : x;
}

// ---------------------------------------------------------------- what a sequence and a tile have to do
// A load whose address is the same in all lanes, through the scalar cache: it is not counted with the vector loads, so nothing
// in flight there has to arrive first.  Nothing writes what is read so (tables) while a kernel here runs.
__device__ __forceinline__ int32_t load_uniform(const int32_t* p)
{
    return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p;
}

struct Seq { int len, n, row0; };      // tokens held, new ones among them, row of the first of these

template <bool STEP> __device__ __forceinline__ Seq sequence(const WkvPagedCall& a, int b)
{
    Seq s;
    s.len = min(max(a.c.lens[b], 0), a.c.max_slots);
    if constexpr (!STEP) {
        const int lo = min(max(a.starts[b], 0), a.n_tokens), hi = min(max(a.starts[b + 1], lo), a.n_tokens);
        s.row0 = lo;
        s.n = min(hi - lo, a.max_new);
    } else {
        s.row0 = b;
        s.n = 1;
    }
    return s;
}

// Keys in the order in which a tile goes over them: the first `first` slots, then those from `lo` on up to the tile's last position,
// both multiples of a block of keys, so that a block is one of slots.
struct Span { int first, lo, blocks, parts, per; };    // (per: blocks of a part, where a part's are next to each other)

__device__ __forceinline__ Span span(const WkvPagedCall& a, int p_lo, int p_hi)
{
    Span s;
    const int low = a.block - 1;                          // (a power of two)
    s.lo = a.c.window > 0 ? max(0, p_lo - a.c.window + 1) & ~low : 0;
    s.first = min((min(a.c.n_sink, s.lo) + low) & ~low, s.lo);
    const int keys = p_hi < 0 ? 0 : s.first + p_hi + 1 - s.lo;
    s.blocks = (keys + low) / a.block;
    // parts of at least a.least blocks; every part has some
    s.parts = max(1, min(a.splits, (s.blocks + a.least - 1) / a.least));
    s.per = max(1, (s.blocks + s.parts - 1) / s.parts);
    if (a.many) s.parts = max(1, (s.blocks + s.per - 1) / s.per);
    return s;
}

struct Tile { int b, h, rows, pos0; Seq q; };    // rows of the unit; position of the first new token

// The unit's sequence; whether it has the row.
template <bool STEP> __device__ __forceinline__ bool unit_of(const WkvPagedCall& a, int unit, int row, Tile& t)
{
    t.b = unit / a.c.kv_heads;
    t.h = unit - t.b * a.c.kv_heads;
    t.q = sequence<STEP>(a, t.b);
    t.rows = t.q.n * a.c.group;
    t.pos0 = t.q.len - t.q.n;
    return row < t.rows;
}

// Chunks of different lengths: K/V head h's tile x of all that there is room for, a tile having a.tile_rows rows.  Sequence b's tiles are those from
// base(b) = starts[b] * group / rows + b on, as many as its rows fill; base(b + 1) is behind the last of them, for the quotient of a sum is at
// most 1 more than the quotients' sum.  The wave looks for b among 64 at a time.  (Of starts that decrease some sequence is found, or none.)
__device__ __forceinline__ bool packed_tile(const WkvPagedCall& a, int h, int x, int& unit, int& tile)
{
    auto base = [&](int b) { return min(max(a.starts[b], 0), a.n_tokens) * a.c.group / a.tile_rows + b; };
    const int lane = threadIdx.x & 63;
    int b = 0, n = a.c.batch;                             // it is one of the n from b on
    while (n > 1) {
        const int step = (n + 63) / 64;
        const int before = __popcll(__ballot(lane * step < n && base(b + min(lane * step, n - 1)) <= x));
        const int k = max(before - 1, 0) * step;
        b += k;
        n = min(step, n - k);
    }
    b = __builtin_amdgcn_readfirstlane(b);
    tile = x - base(b);
    unit = b * a.c.kv_heads + h;
    return (unsigned)tile < (unsigned)((a.max_new * a.c.group + a.tile_rows - 1) / a.tile_rows);
}

// Tokens [first, last) of the unit's sequence into their pages, where those are there.
template <int ROW_BYTES, int THREADS>
__device__ __forceinline__ void append_rows(const WkvPagedCall& a, const Tile& t, int first, int last)
{
    constexpr int PIECES = ROW_BYTES / 16;
    const WkvPages& c = a.c;
    for (int i = first * PIECES + (int)threadIdx.x; i < last * PIECES; i += THREADS) {
        const int token = i / PIECES, x = i % PIECES * 16, pos = t.pos0 + token;
        if (pos < 0) continue;
        const int page = c.table[t.b * c.table_stride + (pos >> c.page_shift)];
        if ((unsigned)page >= (unsigned)c.n_pages) continue;
        const int64_t to = page * c.page_bytes + (pos & ((1 << c.page_shift) - 1)) * c.slot_bytes + t.h * c.head_bytes + x;
        const u32x4_t k = *reinterpret_cast<const u32x4_t*>(a.k_new + (t.q.row0 + token) * a.k_bytes + t.h * a.k_head + x);
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(a.v_new + (t.q.row0 + token) * a.v_bytes + t.h * a.v_head + x);
        *reinterpret_cast<u32x4_t*>(c.k + to) = k;
        *reinterpret_cast<u32x4_t*>(c.v + to) = v;
    }
}

}  // namespace

#endif
