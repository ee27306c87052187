// Eviction from the paged cache by accumulated attention weight (wkv_paged_evict in include/wkv.h).
//
//   wkv_evict_select  a workgroup per unit (sequence, K/V head) finds the slots that stay: the score of the last one that leaves by
//                     three passes of a radix selection over the scores' bits, then the slots in order, counted and written.
//   wkv_evict_move    rows move up within their pages.  Slot i receives what was in list[i] >= i, so a workgroup that goes upwards,
//                     reading a stretch before it writes it, overwrites nothing that is still needed; workgroups share out K, V
//                     and pieces of the rows, which do not touch each other.  The sums move the same way.
//
// 4 x 32768 slots of 8 heads of 128 to 2048, fp16: select 23.6 us (a unit's scores on one compute unit, in registers: three counts by LDS atomics,
// four barriers each, and the list; 4 MB of scores would take 1), move 13.8 us for 37 MB read and 38 MB written, by 288 workgroups, each once
// through the chain list, rows, writes.
// 5 x up to 1237 slots of 12 heads of 64 to 255: 9.0 + 4.3 us.
#include "../../include/wkv.h"
#include "wkv_internal.h"
#include "wkv_device.h"

#include <algorithm>

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int BITS[3] = {11, 11, 10}, BINS = 1 << 11, COPIES = 4;
// Scores as integers of the same order; a NaN is above +inf, -0 is 0.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 0xFF800000u;             // as +inf
    if (b == 0x80000000u) return 0x80000000u;
    return (b >> 31) ? ~b : b | 0x80000000u;
}

// HELD: scores that a thread holds.
template <int HELD>
__global__ __launch_bounds__(THREADS)
void wkv_evict_select_kernel(const WkvPages c, int budget, int list_stride, int recent, int32_t* __restrict__ kept,
                             int32_t* __restrict__ plan, int32_t* __restrict__ list)
{
    constexpr int STRETCH = HELD * THREADS;
    __shared__ __attribute__((aligned(16))) uint32_t s_hist[BINS][COPIES];         // (a lane counts into one of the copies: fewer meet at an address)
    __shared__ uint32_t s_wave[WAVES];
    __shared__ uint32_t s_found[2];
    __shared__ uint64_t s_count[HELD * WAVES], s_total[(HELD * WAVES + 63) / 64];
    const int unit = blockIdx.x, b = unit / c.kv_heads, h = unit - b * c.kv_heads;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int len = min(max(c.lens[b], 0), c.max_slots);
    const float* score = c.scores + (int64_t)unit * c.score_stride;
    int32_t* mine = list + (int64_t)unit * list_stride;
    int32_t* out = kept ? kept + (int64_t)unit * budget : nullptr;

    bool missing = false;
    for (int i = tid; i < (len + (1 << c.page_shift) - 1) >> c.page_shift; i += THREADS)
        missing |= (unsigned)c.table[b * c.table_stride + i] >= (unsigned)c.n_pages;
    missing = __syncthreads_or(missing);
    const bool whole = missing || len <= budget;
    if (h == 0 && tid == 0) { plan[2 * b] = len; plan[2 * b + 1] = whole ? len : budget; }
    if (whole) {
        if (out)
            for (unsigned i = tid; i < (unsigned)budget; i += THREADS) out[i] = !missing && (int)i < len ? (int)i : -1;      // (a budget may be 2^31 - 1)
        return;
    }

    // Slots [first, last) may leave; `want` of them do.  Scores are held in registers, a stretch of the sequence at a time, as integers;
    // slots that stay anyway, and places behind the last slot, are above all (no score is).
    const int first = c.n_sink, last = len - recent, want = len - budget;
    constexpr uint32_t STAYS = ~0u;
    uint32_t x[HELD];
    // (all loads first, from places that are there: a branch around each would wait for each)
    auto hold = [&](int from) {
#pragma unroll
        for (int k = 0; k < HELD; ++k) x[k] = __builtin_bit_cast(uint32_t, score[min(from + k * THREADS + tid, len - 1)]);
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            const int j = from + k * THREADS + tid;
            x[k] = j >= first && j < last ? order_of(__builtin_bit_cast(float, x[k])) : STAYS;
        }
    };
    const bool once = len <= STRETCH;
    if (once) hold(0);
    uint32_t prefix = 0, rest = want;              // bits of the want-th lowest score found so far; its place among those that share them
    int shift = 32;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const uint32_t taken = pass == 0 ? 0u : ~0u << shift;            // the bits that prefix has
        shift -= BITS[pass];
        const uint32_t mask = (1u << BITS[pass]) - 1;
        for (int i = tid; i < BINS; i += THREADS) *reinterpret_cast<uint4*>(s_hist[i]) = make_uint4(0, 0, 0, 0);
        __syncthreads();
        for (int from = 0; from < len; from += STRETCH) {
            if (!once) hold(from);
#pragma unroll
            for (int k = 0; k < HELD; ++k)
                if (from + k * THREADS < len && (pass == 0 || (x[k] & taken) == prefix)) atomicAdd(&s_hist[(x[k] >> shift) & mask][lane % COPIES], 1u);
        }
        __syncthreads();
        // two bins a thread: running count, and the bin in which it reaches `rest`
        const uint4 h0 = *reinterpret_cast<const uint4*>(s_hist[2 * tid]), h1 = *reinterpret_cast<const uint4*>(s_hist[2 * tid + 1]);
        const uint32_t n0 = h0.x + h0.y + h0.z + h0.w, n1 = h1.x + h1.y + h1.z + h1.w;
        uint32_t run = n0 + n1;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t y = __shfl_up(run, d);
            if (lane >= d) run += y;
        }
        if (lane == 63) s_wave[wave] = run;
        __syncthreads();
        uint32_t before = run - n0 - n1;
        for (int w = 0; w < wave; ++w) before += s_wave[w];
        if (before < rest && rest <= before + n0) { s_found[0] = 2 * tid; s_found[1] = before; }
        else if (before + n0 < rest && rest <= before + n0 + n1) { s_found[0] = 2 * tid + 1; s_found[1] = before + n0; }
        __syncthreads();
        prefix |= s_found[0] << shift;
        rest -= s_found[1];
        __syncthreads();
    }
    // Scores below `prefix` leave, and the first `rest` of those equal to it.  The 64 slots of a wave at a time are counted, the counts (those
    // below in the upper half, equal ones in the lower) summed up in the order of the slots, and then it is known where a slot goes.
    const unsigned long long under = (1ull << lane) - 1;
    uint64_t ahead = 0;                            // of the stretches before
    for (int from = 0; from < len; from += STRETCH) {
        if (!once) hold(from);
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            const int less = __popcll(__ballot(x[k] < prefix)), ties = __popcll(__ballot(x[k] == prefix));
            if (lane == 0) s_count[k * WAVES + wave] = (uint64_t)less << 32 | (uint32_t)ties;
        }
        __syncthreads();
        uint64_t n = 0, run = 0;
        if (tid < HELD * WAVES) {
            n = run = s_count[tid];
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint64_t y = (uint64_t)__shfl_up((unsigned long long)run, d);
                if (lane >= d) run += y;
            }
            if (lane == 63) s_total[wave] = run;
        }
        __syncthreads();
        if (tid < HELD * WAVES) {
            uint64_t before = ahead + run - n;
            for (int w = 0; w < wave; ++w) before += s_total[w];
            s_count[tid] = before;
        }
        for (int w = 0; w < (HELD * WAVES + 63) / 64; ++w) ahead += s_total[w];
        __syncthreads();
        const uint64_t before = s_count[min(lane, HELD - 1) * WAVES + wave];      // lane k: of the wave's k-th 64 slots
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            if (from + k * THREADS >= len) break;
            const int j = from + k * THREADS + tid, j0 = from + k * THREADS + wave * 64;
            const int gone = __builtin_amdgcn_readlane((int)(before >> 32), k), tied = __builtin_amdgcn_readlane((int)(uint32_t)before, k);
            bool stays = x[k] > prefix;
            const unsigned long long tb = __ballot(x[k] == prefix);
            if (tb != 0) stays |= x[k] == prefix && tied + __popcll(tb & under) >= (int)rest;
            if (from + (k + 1) * THREADS > len) stays &= j < len;
            const unsigned long long sb = __ballot(stays);
            const int i = __builtin_amdgcn_mbcnt_hi((uint32_t)(sb >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)sb, j0 - gone - min(tied, (int)rest)));
            if (stays) mine[i] = j;
        }
        __syncthreads();
    }
}

// What the workgroup has read is there before any of it writes.
__device__ __forceinline__ void read_then_write()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Workgroups of a unit: K's pieces, V's pieces, the sums (and the list of what stayed, for the caller).  Units run first, in eights, so
// that a unit's workgroups are on one of the chip's eight partitions: two pieces share a cache line.
template <int PIECE>
__global__ __launch_bounds__(THREADS)
void wkv_evict_move_kernel(const WkvPages c, int list_stride, int pieces, int eights, int budget, int32_t* __restrict__ kept, const int32_t* __restrict__ plan, const int32_t* __restrict__ list,
                           int32_t* __restrict__ new_lens, float* new_scores)
{
    const int what = blockIdx.x / eights, unit = blockIdx.x - what * eights;
    if (unit >= c.batch * c.kv_heads) return;
    const int b = unit / c.kv_heads, h = unit - b * c.kv_heads;
    const int tid = threadIdx.x;
    const int len = plan[2 * b], left = plan[2 * b + 1];
    const int32_t* mine = list + (int64_t)unit * list_stride;
    if (what == 2 * pieces) {
        const float* from = c.scores + (int64_t)unit * c.score_stride;
        float* to = new_scores + (int64_t)unit * c.score_stride;
        if (h == 0 && tid == 0) new_lens[b] = left;
        if (kept && left != len)
            for (int i = tid; i < budget; i += THREADS) kept[(int64_t)unit * budget + i] = mine[i];
        constexpr int N = 4;
        for (int i0 = 0; i0 < left; i0 += N * THREADS) {
            float x[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int i = i0 + k * THREADS + tid;
                if (i < left) x[k] = from[left == len ? i : mine[i]];
            }
            read_then_write();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int i = i0 + k * THREADS + tid;
                if (i < left) to[i] = x[k];
            }
        }
        __syncthreads();
        for (int i = left + tid; i < len; i += THREADS) to[i] = 0.f;
        return;
    }
    if (left == len) return;
    char* base = (what < pieces ? c.k : c.v) + h * c.head_bytes + (what % pieces) * PIECE;
    constexpr int LANES = PIECE / 16, ROWS = THREADS / LANES, N = 8;       // rows of a load, loads in flight
    const int row = tid / LANES, off = (tid % LANES) * 16;
    const int in_page = (1 << c.page_shift) - 1;
    const int32_t* table = c.table + b * c.table_stride;
    auto place = [&](int slot) { return base + table[slot >> c.page_shift] * c.page_bytes + (slot & in_page) * c.slot_bytes + off; };
    for (int i0 = 0; i0 < left; i0 += N * ROWS) {
        u32x4_t x[N];
        int src[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int i = i0 + k * ROWS + row;
            src[k] = i < left ? mine[i] : i;
        }
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (src[k] != i0 + k * ROWS + row) x[k] = *reinterpret_cast<const u32x4_t*>(place(src[k]));
        read_then_write();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int i = i0 + k * ROWS + row;
            if (src[k] != i) *reinterpret_cast<u32x4_t*>(place(i)) = x[k];
        }
    }
}

}  // namespace

hipError_t wkv_launch_paged_evict(const WkvPages& c, int row_bytes, int budget, int recent, int32_t* new_lens, float* new_scores,
                                  int32_t* kept, int32_t* plan, int32_t* list, hipStream_t stream)
{
    // (pieces of 128 bytes leave half the chip idle where there are few units: 4 x 32768 slots of 8 heads to 2048: 18.5 us, 13.5 of 64)
    constexpr int PIECE = WKV_EVICT_PIECE;
    const int units = c.batch * c.kv_heads, pieces = row_bytes / PIECE, list_stride = std::min(budget, c.max_slots);
    const int eights = (units + 7) / 8 * 8;
    // (sequences of up to 4096 slots: 8 us with 4 scores a thread, 17 with 32)
    const hipError_t e = wkv_launch(c.max_slots <= 4 * THREADS ? &wkv_evict_select_kernel<4> : &wkv_evict_select_kernel<32>, units, THREADS, stream, c, budget,
                                    list_stride, recent, kept, plan, list);
    if (e != hipSuccess) return e;
    return wkv_launch(&wkv_evict_move_kernel<PIECE>, (unsigned)wkv_evict_groups(units, row_bytes), THREADS, stream, c, list_stride, pieces, eights, budget, kept,
                      (const int32_t*)plan, (const int32_t*)list, new_lens, new_scores);
}
