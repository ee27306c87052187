// Attention of many new tokens over the paged cache (wkv_paged_prefill in include/wkv.h), 16-bit formats.
//
// A workgroup of four waves takes 128 rows of a unit (row r: token r / group, head r % group) and goes over the keys that they see, or
// a part of them, in blocks of 64 or 32.  K and V of a block travel from their pages straight into LDS, the next block's
// while one is used.  A wave has 32 rows: S^T = K Q^T on the 32 x 32 x 16 instruction, whose result holds in a lane four consecutive keys
// of one row at a time, as O^T = V^T P^T takes them for its second operand: weights stay in their lane.  The values' operand, eight keys
// of one element, is read from LDS transposed.  A softmax with a running reference: the sums are scaled down only where a logit
// exceeds the reference by more than 8 octaves (fp16: 15, with a reference 12 below the logit that sets it).
//
// Bound by the matrix and the vector instructions (exponentials, maxima, conversions of the logits), and by the clock, which falls to 1.8 GHz as
// both fill: 4 x 4096 tokens, 32 heads on 8 of 128, fp16: 645 us, 852 TFLOP/s, the matrix units busy 45 % of the cycles, LDS 23 %, none of these
// waiting for a bank; bf16, which does not look for small weights, 575 us; window 1024 over 2 x 8192, bf16, 320 us.  What is read once comes from memory
// 1.2 times (233 MB of 201).
// (A first kernel of 16 rows a workgroup took 2679 us.)
#include "../../include/wkv.h"
#include "wkv_internal.h"
#include "wkv_device.h"
#include "wkv_paged_device.h"

#include <algorithm>
#include <type_traits>

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

constexpr int WAVES = 4, THREADS = 64 * WAVES, WAVE_ROWS = 32, TILE_ROWS = WAVES * WAVE_ROWS;

template <class TT> __device__ __forceinline__ f32x16_t mfma32(u32x4_t a, u32x4_t b, f32x16_t c)
{
    if constexpr (__is_same(TT, TF16))
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// What the values of keys that no row sees are taken from: whatever those hold, a weight of 0 times it has to be 0.
__device__ __attribute__((aligned(16))) uint32_t zero_row[4];

// 16 bytes of every lane from base + off (or from its own address) to 1 KiB of LDS, lane after lane.  Written out because the compiler
// makes reads of LDS wait for all such loads that are under way.  They have no result in registers, and arrive() below waits for them.
// (Nothing else here uses m0.)  LDS is addressed by number.
template <class X> __device__ __forceinline__ const __attribute__((address_space(3))) X* lds_ptr(uint32_t at)
{
    return (const __attribute__((address_space(3))) X*)(uintptr_t)at;
}
__device__ __forceinline__ void load_lds(const char* base, uint32_t off, uint32_t lds)
{
    const uint64_t b = (uint64_t)base;                    // (the same in all lanes, and so that the compiler knows)
    base = (const char*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)b));
    lds = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load_lds(const char* from, uint32_t lds)
{
    lds = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory");
}

template <int D, int KEYS> struct Block {
    static constexpr int BK = KEYS;
    static constexpr int CHUNKS = D / 8;                   // 16-byte pieces of a row
    static constexpr int RPL = 64 / CHUNKS;                // rows of a load (64 lanes, 16 bytes each)
    static constexpr int LOADS = BK / RPL / WAVES;         // loads of a wave
    static constexpr int BYTES = BK * D * 2;
    // The pieces of a row are stored at place (piece ^ turn), so that what is read together lies in different banks of the 64: a piece of 16
    // consecutive keys (K), four pieces next to each other of 4 consecutive keys (V).
    static constexpr int turn_k(int key) { return D == 64 ? key >> 1 & 7 : key & 15; }
    static constexpr int turn_v(int key) { return D == 64 ? (key >> 1 & 1) << 2 : (key & 3) << 2; }
};

// BK: keys of a block, 64 or 32.  With 32 and rows of 256 bytes three workgroups share a compute unit (167 registers, 32 KB), with 64 two (207 to 222): the
// first is ahead where there are that many (us with 64 | 32, bf16: 4 x 4096 tokens 582 | 564, window 1024 over 2 x 8192 366 | 313; fp16 636 | 634, 395 | 348),
// the other where not (2048 tokens, bf16 60 | 70, fp16 66 | 80).
template <class TT, int D, int BK>
__global__ __launch_bounds__(THREADS, D * BK > 4096 ? 2 : 3)
void wkv_paged_flash_kernel(const WkvPagedCall a, int tiles, int spread)
{
    using B = Block<D, BK>;
    constexpr int NB = BK / 32, KS = D / 16, DB = D / 32;
    // The reference may be LAG below a row's largest logit.  In fp16 it is lower by RAISED more, so that weights go up to 2^15, what the format can hold, and
    // lose bits below SMALL only; with a smaller LAG that is further from the largest.
    constexpr bool NARROW = __is_same(TT, TF16);
    constexpr float LAG = NARROW ? 3.f : 8.f, RAISED = NARROW ? 12.f : 0.f, SMALL = 0x1p-14f, MORE = 0x1p29f;
    __shared__ __attribute__((aligned(1024))) char s_kv[4 * B::BYTES];
    const uint32_t s_k0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_kv, s_v0 = s_k0 + B::BYTES;
    const uint32_t s_k1 = s_k0 + 2 * B::BYTES, s_v1 = s_k0 + 3 * B::BYTES;

    // Workgroups are dealt to the chip's eight partitions in turn: with spread, all of a unit's go to one of them, whose cache then
    // holds the unit's K and V.  Tiles far into the sequence, which have the most keys, come first.
    int id = blockIdx.x, unit, tile, part = 0;
    const int per_unit = tiles * a.splits;
    if (a.slots > 0) {
        // (a K/V head's on one partition where there are 8 of them, or 16, ...)
        if (!packed_tile(a, id % a.c.kv_heads, a.slots - 1 - id / a.c.kv_heads, unit, tile)) return;
    } else if (spread) {
        const int x = id & 7;
        id >>= 3;
        unit = id / per_unit * 8 + x;
        id = id % per_unit;
    } else {
        unit = id / per_unit;
        id = id % per_unit;
    }
    if (a.slots == 0) {
        part = id % a.splits;
        tile = tiles - 1 - id / a.splits;
    }
    Tile t;
    if (!unit_of<false>(a, unit, tile * TILE_ROWS, t)) return;
    const WkvPages& c = a.c;
    const int group = c.group;
    const int r0 = tile * TILE_ROWS, r1 = min(t.rows, r0 + TILE_ROWS);
    const int t_lo = t.pos0 + r0 / group, t_hi = t.pos0 + (r1 - 1) / group;       // positions of the tile's tokens
    const Span sp = span(a, t_lo, t_hi);
    if (part >= sp.parts) return;
    const int begin = part * sp.per, end = min(sp.blocks, begin + sp.per);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half_q = lane >> 5;
    const int window = c.window > 0 ? c.window : 0x40000000;
    const int in_page = (1 << c.page_shift) - 1;

    // the lane's row, and the positions of the wave's
    const int w0 = r0 + wave * WAVE_ROWS;
    const int row_q = min(w0 + col, r1 - 1), token_q = row_q / group;
    const int p_row = w0 + col < r1 ? t.pos0 + token_q : -1;
    const int p_lo = t.pos0 + min(w0, r1 - 1) / group, p_hi = t.pos0 + (min(w0 + WAVE_ROWS, r1) - 1) / group;
    u32x4_t q[KS];
    {
        const char* src = a.q + (t.q.row0 + token_q) * a.q_bytes + (t.h * group + row_q - token_q * group) * a.q_head + half_q * 16;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const u32x4_t*>(src + s * 32);
    }

    const int32_t* table = c.table + t.b * c.table_stride;
    auto slot_of = [&](int blk) { const int i = blk * BK; return __builtin_amdgcn_readfirstlane(i < sp.first ? i : i - sp.first + sp.lo); };
    constexpr int NG = BK / 16;
    // pages of a block's stretches of 16 slots, as the table says
    auto entries = [&](int pos, int (&e)[NG]) {
#pragma unroll
        for (int i = 0; i < NG; ++i) e[i] = load_uniform(table + min((pos + i * 16) >> c.page_shift, c.max_pages - 1));
    };
    // -1 for what is none
    auto known = [&](int pos, int (&e)[NG]) {
#pragma unroll
        for (int i = 0; i < NG; ++i) e[i] = (unsigned)e[i] < (unsigned)c.n_pages && pos + i * 16 < c.max_slots ? e[i] : -1;
    };
    auto all_there = [&](const int (&e)[NG]) {
        bool x = true;
#pragma unroll
        for (int i = 0; i < NG; ++i) x &= e[i] >= 0;
        return x;
    };

    const char* kh = c.k + t.h * c.head_bytes;
    const char* vh = c.v + t.h * c.head_bytes;
    // The call's own tokens, from slot `fresh` on, are read from where they are; the tile's workgroup also puts its tokens' rows into their pages,
    // which nothing here reads.
    const int fresh = a.k_new ? t.pos0 : 0x7FFFFFFF;
    const char* kf = a.k_new + t.h * a.k_head + (t.q.row0 - t.pos0) * a.k_bytes;
    const char* vf = a.v_new + t.h * a.v_head + (t.q.row0 - t.pos0) * a.v_bytes;
    if (a.k_new && part == 0) append_rows<D * 2, THREADS>(a, t, (r0 + group - 1) / group, min(t.q.n, (r0 + TILE_ROWS + group - 1) / group));

    auto load = [&](uint32_t kb, uint32_t vb, int pos, const int (&pages)[NG]) __attribute__((always_inline)) {
        // every key is one that some row of the tile sees, or at least a finite one
        const bool inside = all_there(pages) && pos + BK - 1 <= t_hi && (pos > t_lo - window || pos + BK <= c.n_sink);
        const uint32_t kl = kb + wave * 1024, vl = vb + wave * 1024;
        int ln = threadIdx.x & 63;                        // (and what follows from it: not kept from block to block)
        if constexpr (D > 128) asm volatile("" : "+v"(ln));
        const int lrow = ln / B::CHUNKS, lpiece = ln % B::CHUNKS;
        // load i: its first row, the lane's, the page (in narrow rows the waves' loads are of two stretches of 16 slots)
        auto first = [&](int i) { return (i * WAVES + wave) * B::RPL; };
        auto page_of = [&](int i) {
            return WAVES * B::RPL > 16 ? (wave * B::RPL >= 16 ? pages[2 * i + 1] : pages[2 * i]) : pages[i * WAVES * B::RPL / 16];
        };
        if (inside && pos + BK <= fresh) {
            const uint32_t down = (uint32_t)(lrow * (int)c.slot_bytes);
#pragma unroll
            for (int i = 0; i < B::LOADS; ++i) {
                const int64_t at = page_of(i) * c.page_bytes + ((pos + first(i)) & in_page) * c.slot_bytes;
                load_lds(kh + at, down + ((lpiece ^ B::turn_k(first(i) + lrow)) * 16), kl + i * (WAVES * 1024));
                load_lds(vh + at, down + ((lpiece ^ B::turn_v(first(i) + lrow)) * 16), vl + i * (WAVES * 1024));
            }
        } else if (inside && pos >= fresh) {
            const uint32_t kd = (uint32_t)(lrow * (int)a.k_bytes), vd = (uint32_t)(lrow * (int)a.v_bytes);
#pragma unroll
            for (int i = 0; i < B::LOADS; ++i) {
                load_lds(kf + (pos + first(i)) * a.k_bytes, kd + ((lpiece ^ B::turn_k(first(i) + lrow)) * 16), kl + i * (WAVES * 1024));
                load_lds(vf + (pos + first(i)) * a.v_bytes, vd + ((lpiece ^ B::turn_v(first(i) + lrow)) * 16), vl + i * (WAVES * 1024));
            }
        } else {
#pragma unroll
            for (int i = 0; i < B::LOADS; ++i) {
                const int page = page_of(i), in = first(i) + lrow, p = pos + in;
                const int64_t at = max(page, 0) * c.page_bytes + (p & in_page) * c.slot_bytes;
                const bool any = page >= 0 && p <= t_hi && (p > t_lo - window || p < c.n_sink), new_row = p >= fresh && p < t.q.len;
                const char* ks = new_row ? kf + p * a.k_bytes : kh + at;
                const char* vs = new_row ? vf + p * a.v_bytes : vh + at;
                vs += (lpiece ^ B::turn_v(in)) * 16;
                load_lds(ks + (lpiece ^ B::turn_k(in)) * 16, kl + i * (WAVES * 1024));
                load_lds(any ? vs : reinterpret_cast<const char*>(zero_row), vl + i * (WAVES * 1024));
            }
        }
    };

    // Where the lane reads: K's piece 2 i + half of key col, V's piece of elements 32 i + (lane & 31) of the key of its four lanes; other
    // keys and pieces are at fixed distances, but for the turn, which flips bits.
    uint32_t k_at = col * (D * 2) + ((half_q ^ B::turn_k(col)) << 4);
    const int v_key = half_q * 4 + ((lane & 15) >> 2);
    uint32_t v_at = v_key * (D * 2) + (((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ B::turn_v(v_key)) << 4) + (lane & 1) * 8;

    float ref = -INFINITY, l = 0.f;       // log2 of the weights' reference; the sum of the lane's weights
    f32x16_t o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.f;

    // S^T of 32 keys
    auto logits = [&](uint32_t k_at, uint32_t kb) __attribute__((always_inline)) {
        f32x16_t s = {};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const u32x4_t k = *lds_ptr<u32x4_t>((k_at ^ (i << 5)) + kb);
            s = mfma32<TT>(k, q[i], s);
        }
        return s;
    };
    // the values' operand of O^T = V^T P^T: 16 keys, elements 32 i and the following
    auto values = [&](uint32_t v_at, uint32_t vb, int i) __attribute__((always_inline)) {
        const uint32_t at = (v_at ^ (i << 6)) + vb;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)lds_ptr<s16x4_t>(at));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)lds_ptr<s16x4_t>(at + 8 * (D * 2)));
        const u32x2_t lw = __builtin_bit_cast(u32x2_t, lo), hw = __builtin_bit_cast(u32x2_t, hi);
        return u32x4_t{lw.x, lw.y, hw.x, hw.y};
    };
    auto scale_all = [&](float f) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] *= f;
    };
    // What rounding to fp16 takes from a weight below SMALL (a logit 18 and more below a row's largest) is up to 2^-25, and so a row's sum may miss the number
    // of such weights times 2^-25 times the largest value.  (That matters where a key takes nearly all of a row and has a value near 0: the output is then
    // left to such weights.)  Blocks that have some are counted, and their largest value is kept; if a row's sums are so small that the loss could be
    // seen in them, the tile goes over its keys a second time, with the small weights by themselves.  4 x 4096 tokens: looking for small weights costs 5 %
    // (612 -> 645 us), queries of 3 times the size, which have some in every block, 800 us (1170 with the small weights by themselves at once); a first
    // key 22 above all others 867, with values of 0 1674.
    [[maybe_unused]] int small_blocks = 0;
    [[maybe_unused]] uint32_t largest = 0;                // two absolute values of fp16, as bits, which are in order
    auto count_small = [&](uint32_t vb) __attribute__((always_inline)) {
        ++small_blocks;
#pragma unroll 2
        for (int i = 0; i < BK * D / 512; ++i) {
            const u32x4_t x = *lds_ptr<u32x4_t>(vb + lane * 16 + i * 1024);
#pragma unroll
            for (int w = 0; w < 4; ++w)
                largest = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, largest), __builtin_bit_cast(u16x2_t, x[w] & 0x7FFF7FFFu)));
        }
    };

    auto use = [&](uint32_t kb, uint32_t vb, int pos, const int (&pages)[NG]) __attribute__((always_inline)) {
        if (pos > p_hi) return;                                            // (the wave's rows are all before it)
        // (addresses made of these are not kept in registers from block to block)
        if constexpr (D > 128) asm("" : "+v"(k_at), "+v"(v_at));
        else if constexpr (NARROW) asm("" : "+v"(k_at));
        f32x16_t s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] = logits(k_at, kb + b * 32 * (D * 2));
        const bool full = all_there(pages) && pos + BK - 1 <= p_lo && (pos > p_hi - window || pos + BK <= c.n_sink);
        if (!full) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int p = pos + b * 32 + (j >> 2) * 8 + half_q * 4 + (j & 3);
                    const bool seen = pages[b * 2 + (j >> 3)] >= 0 && p <= p_row && (p > p_row - window || p < c.n_sink);
                    s[b][j] = seen ? s[b][j] : -INFINITY;
                }
        }
        [[maybe_unused]] float low = INFINITY;            // the lowest logit that is seen, of a block that is not full
        if constexpr (NARROW)
            if (!full) {
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int j = 0; j < 16; ++j) low = fminf(low, s[b][j] == -INFINITY ? INFINITY : s[b][j]);
            }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[b][j]);
        {
            float x0, x1;
            lane_pair<32>(top, x0, x1);
            top = fmaxf(x0, x1) * a.scale;
        }
        if (__any(top > ref + (LAG + RAISED))) {
            const float now = fmaxf(ref, top - RAISED);
            const float f = ref == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - now);
            ref = now;
            l *= f;
            scale_all(f);
        }
        const float minus = ref == -INFINITY ? 0.f : -ref;
        [[maybe_unused]] const bool edge = NARROW && !full && __any(__builtin_fmaf(low, a.scale, minus) < -14.f);
        [[maybe_unused]] float least = MORE;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                s[b][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j], a.scale, minus));
                l += s[b][j];
                if constexpr (NARROW) least = fminf(least, s[b][j]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {                                  // 16 keys each
                // weights rounded to the format: off by half a step each, and so is the output by half a step of sum w |v|
                u32x4_t p;
#pragma unroll
                for (int w = 0; w < 4; ++w) p[w] = pack2<TT>(s[b][j * 8 + 2 * w], s[b][j * 8 + 2 * w + 1]);
#pragma unroll
                for (int i = 0; i < DB; ++i) o[i] = mfma32<TT>(values(v_at, vb + (b * 32 + j * 16) * (D * 2), i), p, o[i]);
            }
        }
        if constexpr (NARROW) {
            asm volatile("" : "+v"(l));                   // (the weights have been added up: they are not kept for it)
            if (__builtin_expect(full ? __any(least < SMALL) : edge, 0)) count_small(vb);
        }
    };

    // Every wave has waited for its own loads of a block when it comes to the barrier, and for what it read of the block before: after it
    // the block is whole, and the other buffer is free for the next.
    auto arrive = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);               // vmcnt(0) lgkmcnt(0), in a form that the compiler counts by
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto sweep = [&](auto&& use) __attribute__((always_inline)) {
        int pos = slot_of(begin), pages[NG], next = 0, after[NG];
        if (begin < end) {
            entries(pos, pages);
            known(pos, pages);
            load(s_k0, s_v0, pos, pages);
            next = slot_of(min(begin + 1, end - 1));
            entries(next, after);
        }
        auto round = [&](int blk, uint32_t k, uint32_t v, uint32_t k_next, uint32_t v_next) __attribute__((always_inline)) {
            arrive();
            known(next, after);
            if (blk + 1 < end) load(k_next, v_next, next, after);
            const int p = pos;
            int e[NG];
#pragma unroll
            for (int i = 0; i < NG; ++i) { e[i] = pages[i]; pages[i] = after[i]; }
            pos = next;
            next = slot_of(min(blk + 2, end - 1));
            entries(next, after);
            use(k, v, p, e);
        };
        for (int blk = begin; blk < end; blk += 2) {
            round(blk, s_k0, s_v0, s_k1, s_v1);
            if (blk + 1 < end) round(blk + 1, s_k1, s_v1, s_k0, s_v0);
        }
    };
    sweep(use);
    l = pair_sum<32>(l);

    if constexpr (NARROW) {
        bool again = false;
        if (small_blocks > 0) {
            uint32_t v = max(largest & 0xFFFF, largest >> 16);
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
            const float lost = (float)(small_blocks * BK) * 0x1p-25f * (float)__builtin_bit_cast(_Float16, (uint16_t)v);
            float top = 0.f, x0, x1;
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) top = fmaxf(top, __builtin_fabsf(o[i][j]));
            lane_pair<32>(top, x0, x1);
            top = fmaxf(x0, x1);
            // half of fp16's smallest step, or a 64th of half a step of the row's largest output
            again = __any(l > 0.f && lost > l * 0x1p-25f && lost > top * 0x1p-18f);
        }
        if (__builtin_expect(__syncthreads_or(again), 0)) {
            // The reference stays as it is now.  What rounding takes from a weight below SMALL goes by itself, raised by MORE: half a step of a weight is left
            // of it down to 2^-55 of a row's largest, and 2^-66 of that one below.
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
            const float minus = ref == -INFINITY ? 0.f : -ref;
            sweep([&](uint32_t kb, uint32_t vb, int pos, const int (&pages)[NG]) __attribute__((always_inline)) {
                if (pos > p_hi) return;
#pragma unroll 1
                for (int b = 0; b < NB; ++b) {
                    uint32_t k_from = k_at, v_from = v_at;
                    asm volatile("" : "+v"(k_from), "+v"(v_from));        // (addresses made of these are not kept in registers)
                    f32x16_t s = logits(k_from, kb + b * 32 * (D * 2));
                    __builtin_amdgcn_sched_barrier(0);    // (one thing after the other, in few registers)
                    u32x4_t p[2], more[2];
#pragma unroll
                    for (int w = 0; w < 8; ++w) {
                        const int page = b ? pages[NG - 2 + (w >> 2)] : pages[w >> 2];
                        float x[2], y[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int j = 2 * w + e, at = pos + b * 32 + (j >> 2) * 8 + half_q * 4 + (j & 3);
                            const int seen = (page >= 0) & (at <= p_row) & ((at > p_row - window) | (at < c.n_sink));
                            x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j], a.scale, minus));
                            x[e] = seen ? x[e] : 0.f;
                        }
                        p[w >> 2][w & 3] = pack2<TT>(x[0], x[1]);
                        unpack2<TT>(p[w >> 2][w & 3], y[0], y[1]);
                        more[w >> 2][w & 3] = pack2<TT>(x[0] < SMALL ? (x[0] - y[0]) * MORE : 0.f, x[1] < SMALL ? (x[1] - y[1]) * MORE : 0.f);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int i = 0; i < DB; ++i) {
                        f32x16_t d = {};
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const u32x4_t v = values(v_from, vb + (b * 32 + j * 16) * (D * 2), i);
                            o[i] = mfma32<TT>(v, p[j], o[i]);
                            d = mfma32<TT>(v, more[j], d);
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[i][j] = __builtin_fmaf(d[j], 1.f / MORE, o[i][j]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            });
        }
    }

    // (the lane's row once more, so that it takes no registers in the loop above)
    int tid = threadIdx.x;
    asm("" : "+v"(tid));
    const int row = w0 + (tid & 31), token = min(row, r1 - 1) / group, head = t.h * group + min(row, r1 - 1) - token * group, half = tid >> 5 & 1;

    // A value that is not finite spoils the sums of rows that do not see it (0 x infinity), and sums of the largest values may overflow.  If one is
    // not finite, the wave forms them anew, key by key: a lane has a row and half of its elements.
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) z = __builtin_fmaf(o[i][j], 0.f, z);
    const bool spoilt = __any(z != 0.f);                                   // (0 x infinity and 0 x NaN are NaN, which is no 0)
    if (spoilt) {
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
        const char* qr = a.q + (t.q.row0 + token) * a.q_bytes + head * a.q_head;
        ref += CAREFUL<TT>;
        l *= __builtin_amdgcn_exp2f(-CAREFUL<TT>);
        const float minus = ref == -INFINITY ? 0.f : -ref;
#pragma unroll 1
        for (int blk = begin; blk < end; ++blk) {
            const int p0 = slot_of(blk);
#pragma unroll 1
            for (int k = 0; k < BK; ++k) {
                const int p = p0 + k;
                if (p >= t.q.len) break;
                const int page = load_uniform(table + (p >> c.page_shift));
                if ((unsigned)page >= (unsigned)c.n_pages) continue;
                const int64_t at = page * c.page_bytes + (p & in_page) * c.slot_bytes;
                const char* kr = p >= fresh ? kf + p * a.k_bytes : kh + at;
                const char* vr = p >= fresh ? vf + p * a.v_bytes : vh + at;
                float dot = 0.f;
#pragma unroll 1
                for (int e = half * (D / 2); e < (half + 1) * (D / 2); ++e) dot += load_elem<TT>(qr, e) * load_elem<TT>(kr, e);
                dot = pair_sum<32>(dot);
                if (p <= p_row && (p > p_row - window || p < c.n_sink)) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(dot, a.scale, minus));
#pragma unroll
                    for (int i = 0; i < DB; ++i)
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[i][j] += w * load_elem<TT>(vr, i * 32 + (j >> 2) * 8 + half * 4 + (j & 3));
                }
            }
        }
    }

    const bool direct = sp.parts == 1, mine = row < r1;
    if (direct) {
        const float inv = l != 0.f ? 1.f / l : 0.f;
        char* dst = a.out + (t.q.row0 + token) * a.out_bytes + head * a.out_head;
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int j = 0; j < 4; j += 2) {                               // elements 8 j .. 8 j + 15 of the 32: halves of a lane pair joined
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    w[k] = pack2<TT>(mean<TT>(o[i][(j + (k >> 1)) * 4 + (k & 1) * 2], inv), mean<TT>(o[i][(j + (k >> 1)) * 4 + (k & 1) * 2 + 1], inv));
                const uint2v_t x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
                const uint2v_t y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
                if (mine) *reinterpret_cast<u32x4_t*>(dst + (i * 32 + (j + half) * 8) * 2) = u32x4_t{x.x, y.x, x.y, y.y};
            }
    } else {
        float* cell = a.part + ((((int64_t)unit * a.tiles + row / ROWS) * a.splits + part) * ROWS + row % ROWS) * D;
        if (mine) {
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<f32x4_t*>(cell + i * 32 + j * 8 + half * 4) = f32x4_t{o[i][j * 4], o[i][j * 4 + 1], o[i][j * 4 + 2], o[i][j * 4 + 3]};
        }
    }
    if (mine && half == 0) {
        if (a.ml) {
            float* ml = a.ml + (((int64_t)unit * a.tiles + row / ROWS) * a.splits + part) * 32 + row % ROWS;
            ml[0] = ref;
            ml[16] = l;
        }
        if (a.lse && direct)
            a.lse[(int64_t)(t.q.row0 + token) * (c.kv_heads * group) + head] = ref == -INFINITY ? INFINITY : ref + __builtin_amdgcn_logf(l);
    }
}

// ---------------------------------------------------------------- weights of a prefill's rows, summed for every slot
//
// sum over the rows of 2^(logit - log-sum-exp).  A wave keeps 32 keys in registers and goes over all rows that see some of
// its workgroup's keys, 64 at a time through LDS: S = Q K^T leaves in a lane 16 rows of one key, so the sums stay in the lane.  Bound by the
// vector instructions: an exponential, a multiply-add and an addition a logit, 24 cycles against the 16 of its matrix instructions.
// (3 x 333 tokens, 32 heads, onto 6001 slots and fewer, bf16: 56 us.)
template <class TT, int D>
__global__ __launch_bounds__(THREADS, 2)
void wkv_paged_colsum_kernel(const WkvPagedCall a, int by_unit, int64_t fast, int64_t first)
{
    constexpr int KS = D / 16, CHUNKS = D / 8, RPL = 64 / CHUNKS, QROWS = 64, LOADS = QROWS / RPL / WAVES, BYTES = QROWS * D * 2;
    __shared__ __attribute__((aligned(1024))) char s_q[2 * BYTES];
    __shared__ __attribute__((aligned(16))) float s_lse[2][QROWS];
    __shared__ __attribute__((aligned(16))) int s_pos[2][QROWS];
    const uint32_t q0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_q;
    const WkvPages& c = a.c;
    // Prompts: the first keys, which the most rows see, of all units first, which spreads the work over the compute units (unit after unit, some got
    // only first keys: 4 x 4096 620 -> 430 us).  Chunks onto longer sequences: unit after unit.
    // A key block's rows are cut into a.row_parts where there are few blocks.
    const int row_part = blockIdx.x % a.row_parts, id = blockIdx.x / a.row_parts;
    const int slow = (int)first + id / (int)fast, quick = id % (int)fast;
    const int unit = by_unit ? slow : quick, k0 = (by_unit ? quick : slow) * (WAVES * 32);
    Tile t;
    if (!unit_of<false>(a, unit, 0, t) || k0 >= t.q.len) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5, group = c.group;
    const int window = c.window > 0 ? c.window : 0x40000000, in_page = (1 << c.page_shift) - 1;

    // the wave's keys
    const int kw = k0 + wave * 32, key = kw + col;
    u32x4_t k[KS];
    const int page = c.table[t.b * c.table_stride + min(key >> c.page_shift, c.max_pages - 1)];
    const bool there = (unsigned)page < (unsigned)c.n_pages && key < t.q.len;
    {
        const char* src = c.k + (there ? page : 0) * c.page_bytes + (key & in_page) * c.slot_bytes + t.h * c.head_bytes + half * 16;
#pragma unroll
        for (int i = 0; i < KS; ++i) k[i] = *reinterpret_cast<const u32x4_t*>(src + i * 32);
    }

    // rows that see some key of the workgroup
    const int i0 = max(0, k0 - t.pos0);
    const int i1 = k0 < c.n_sink ? t.q.n : (int)min((int64_t)t.q.n, (int64_t)k0 + WAVES * 32 - 1 + window - t.pos0);
    int r_lo = i0 * group & -QROWS, r_hi = i1 * group;
    if (a.row_parts > 1) {
        const int each = ((r_hi - r_lo + QROWS - 1) / QROWS + a.row_parts - 1) / a.row_parts * QROWS;
        r_lo += row_part * each;
        r_hi = min(r_hi, r_lo + each);
    }
    // Where the lane's rows of a load are: from one tile to the next a fixed distance on, where the group's size divides QROWS
    const bool even = QROWS % group == 0;
    const int lrow = lane / CHUNKS, piece = lane % CHUNKS;
    const char* qh = a.q + t.q.row0 * a.q_bytes + (int64_t)t.h * group * a.q_head;
    auto row_at = [&](int row) {                             // (rows behind the last one: that one again, with a weight of 0)
        const int r = min(row, t.rows - 1), token = r / group;
        return qh + token * a.q_bytes + (r - token * group) * a.q_head;
    };
    const char* at[LOADS];
    if (r_lo < r_hi)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) at[i] = row_at(r_lo + (i * WAVES + wave) * RPL + lrow);
    auto load = [&](uint32_t q, int r0) {
        const bool known = even && r0 + QROWS <= t.rows;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = (i * WAVES + wave) * RPL + lrow;
            if (!known) at[i] = row_at(r0 + r);
            load_lds(at[i] + ((piece ^ Block<D, 32>::turn_k(r)) * 16), q + (i * WAVES + wave) * 1024);
            at[i] += QROWS / group * a.q_bytes;
        }
    };
    float lse = INFINITY;
    int pos = -1;
    auto load_row = [&](int r0) {
        lse = INFINITY;
        pos = -1;
        const int row = r0 + threadIdx.x, token = row / group;
        if (threadIdx.x < QROWS && row < t.rows) {
            lse = a.lse[(int64_t)(t.q.row0 + token) * (c.kv_heads * group) + t.h * group + row - token * group];
            pos = t.pos0 + token;
        }
    };
    auto keep_row = [&](int x) {
        if (threadIdx.x < QROWS) { s_lse[x][threadIdx.x] = lse; s_pos[x][threadIdx.x] = pos; }
    };

    const uint32_t q_at = col * (D * 2) + ((half ^ Block<D, 32>::turn_k(col)) << 4);
    float sum = 0.f;
    auto add = [&](uint32_t q, int x, auto full) {
#pragma unroll
        for (int rb = 0; rb < QROWS / 32; ++rb) {
            u32x4_t f[KS];
#pragma unroll
            for (int i = 0; i < KS; ++i) f[i] = *lds_ptr<u32x4_t>((q_at ^ (i << 5)) + q + rb * 32 * (D * 2));
            f32x16_t s = {};
#pragma unroll
            for (int i = 0; i < KS; ++i) s = mfma32<TT>(f[i], k[i], s);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4_t ls = *reinterpret_cast<const f32x4_t*>(&s_lse[x][rb * 32 + j * 8 + half * 4]);
                const int4 pr = *reinterpret_cast<const int4*>(&s_pos[x][rb * 32 + j * 8 + half * 4]);
                const int p4[4] = {pr.x, pr.y, pr.z, pr.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j * 4 + e], a.scale, -ls[e]));
                    if constexpr (!decltype(full)::value) {
                        asm("" : "+v"(w));                    // (a selection, no branch: w may be NaN)
                        w = key <= p4[e] && (key > p4[e] - window || key < c.n_sink) ? w : 0.f;
                    }
                    sum += w;
                }
            }
        }
    };
    auto use = [&](uint32_t q, int x, int r0) {
        // positions of the tile's first and last row
        const int p_lo = t.pos0 + r0 / group, p_hi = t.pos0 + (min(r0 + QROWS, t.rows) - 1) / group;
        if (kw > p_hi) return;
        if (kw + 31 <= p_lo && (kw > p_hi - window || kw + 32 <= c.n_sink)) add(q, x, std::true_type{});
        else add(q, x, std::false_type{});
    };
    auto arrive = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0F70);               // vmcnt(0)
        __syncthreads();
        asm volatile("" ::: "memory");
    };
    if (r_lo < r_hi) {
        load(q0, r_lo);
        load_row(r_lo);
        keep_row(0);
        for (int r0 = r_lo, x = 0; r0 < r_hi; r0 += QROWS, x ^= 1) {
            arrive();
            const bool more = r0 + QROWS < r_hi;
            if (more) {
                load(q0 + (x ^ 1) * BYTES, r0 + QROWS);
                load_row(r0 + QROWS);
            }
            use(q0 + x * BYTES, x, r0);
            if (more) keep_row(x ^ 1);
        }
    }
    sum = pair_sum<32>(sum);
    if (half == 0 && key < t.q.len && a.row_parts > 1)
        a.colsums[((int64_t)row_part * c.batch * c.kv_heads + unit) * a.logit_stride + key] = there ? sum : 0.f;
    else if (half == 0 && key < t.q.len) {
        float* sc = c.scores + (int64_t)unit * c.score_stride + key;
        if (a.k_new && key >= t.pos0) *sc = there ? sum : 0.f;
        else if (there) *sc += sum;
    }
}

// The row parts' sums added to the scores, in the order of the parts.
__global__ __launch_bounds__(THREADS)
void wkv_paged_colsum_join_kernel(const WkvPagedCall a, int per_unit)
{
    const WkvPages& c = a.c;
    const int unit = blockIdx.x / per_unit, key = blockIdx.x % per_unit * THREADS + threadIdx.x;
    Tile t;
    if (!unit_of<false>(a, unit, 0, t) || key >= t.q.len) return;
    const int page = c.table[t.b * c.table_stride + (key >> c.page_shift)];
    const bool there = (unsigned)page < (unsigned)c.n_pages, fresh = a.k_new && key >= t.pos0;
    float* sc = c.scores + (int64_t)unit * c.score_stride + key;
    float w = 0.f;
    for (int i = 0; i < a.row_parts; ++i) w += a.colsums[((int64_t)i * c.batch * c.kv_heads + unit) * a.logit_stride + key];
    if (fresh) *sc = w;
    else if (there) *sc += w;
}

}  // namespace

int wkv_paged_row_parts(int64_t units, int64_t slots, int64_t rows)
{
    // about 1024 workgroups, of at least 4 tiles of 64 rows each
    return (int)std::max<int64_t>(1, std::min<int64_t>({1024 / (units * ((slots + 127) / 128)), rows / 256, 8}));
}

hipError_t wkv_launch_paged_colsum(const WkvPagedCall& a, int dtype, int head_dim, hipStream_t stream)
{
    const int64_t units = (int64_t)a.c.batch * a.c.kv_heads;
    const int64_t blocks = (a.c.max_slots + WAVES * 32 - 1) / (WAVES * 32);
    const int by_unit = a.max_new < a.c.max_slots / 2;
    const int64_t fast = by_unit ? blocks : units, all = by_unit ? units : blocks;      // the index that runs first, the other
    const int64_t most = std::max<int64_t>(1, ((1 << 24) - 1) / (fast * a.row_parts));
    auto go = [&](auto t, auto d) {
        using TT = decltype(t);
        constexpr int D = decltype(d)::value;
        for (int64_t b = 0; b < all;) {                 // in pieces below 2^32 threads
            const int64_t n = std::min<int64_t>(all - b, most);
            const hipError_t e = wkv_launch(&wkv_paged_colsum_kernel<TT, D>, (unsigned)(n * fast * a.row_parts), THREADS, stream, a, by_unit, fast, b);
            if (e != hipSuccess) return e;
            b += n;
        }
        if (a.row_parts == 1) return hipSuccess;
        const int per_unit = (a.c.max_slots + THREADS - 1) / THREADS;
        return wkv_launch(&wkv_paged_colsum_join_kernel, (unsigned)(units * per_unit), THREADS, stream, a, per_unit);
    };
    auto size = [&](auto t) {
        return head_dim == 64 ? go(t, std::integral_constant<int, 64>{}) : head_dim == 128 ? go(t, std::integral_constant<int, 128>{})
                                                                                           : go(t, std::integral_constant<int, 256>{});
    };
    return dtype == WKV_FP16 ? size(TF16{}) : size(TBF16{});
}

hipError_t wkv_launch_paged_flash(const WkvPagedCall& a, int dtype, int head_dim, hipStream_t stream)
{
    const int units = a.c.batch * a.c.kv_heads, tiles = (a.tiles * ROWS + TILE_ROWS - 1) / TILE_ROWS;
    const int spread = units % 8 == 0;
    auto go = [&](auto t, auto d, auto bk) {
        using TT = decltype(t);
        constexpr int D = decltype(d)::value, BK = decltype(bk)::value;
        return wkv_launch(&wkv_paged_flash_kernel<TT, D, BK>, (unsigned)wkv_paged_groups(a), THREADS, stream, a, tiles, spread);
    };
    auto wide = [&](auto t) {
        constexpr std::integral_constant<int, 32> few{};
        constexpr std::integral_constant<int, 64> d64{}, many{};
        constexpr std::integral_constant<int, 128> d128{};
        if (head_dim == 64) return go(t, d64, many);
        if (head_dim == 128) return a.block == 64 ? go(t, d128, many) : go(t, d128, few);
        return go(t, std::integral_constant<int, 256>{}, few);
    };
    return dtype == WKV_FP16 ? wide(TF16{}) : wide(TBF16{});
}
