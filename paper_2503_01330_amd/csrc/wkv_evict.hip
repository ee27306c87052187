// Eviction from the paged cache by accumulated attention weight (wkv_paged_evict in include/wkv.h).
//
//   wkv_evict_select  a workgroup per unit (sequence, K/V head) finds the slots that stay: the score of the last one that leaves by
//                     three passes of a radix selection over the scores' bits, then the slots in order, counted and written.
//   wkv_evict_move    rows move up within their pages.  Slot i receives what was in list[i] >= i, so a workgroup that goes upwards,
//                     reading a stretch before it writes it, overwrites nothing that is still needed; workgroups share out K, V
//                     and pieces of the rows, which do not touch each other.  The sums move the same way.
#include "../../include/wkv.h"
#include "wkv_internal.h"
#include "wkv_device.h"

#include <algorithm>

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int BITS[3] = {11, 11, 10}, BINS = 1 << 11;

// Scores as integers of the same order; a NaN is above +inf, -0 is 0.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 0xFF800000u;             // as +inf
    if (b == 0x80000000u) return 0x80000000u;
    return (b >> 31) ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(THREADS)
void wkv_evict_select_kernel(const WkvPages c, int budget, int list_stride, int recent, int32_t* __restrict__ kept,
                             int32_t* __restrict__ plan, int32_t* __restrict__ list)
{
    __shared__ uint32_t s_hist[BINS];
    __shared__ uint32_t s_wave[WAVES];
    __shared__ uint32_t s_found[2];
    __shared__ int s_less[WAVES], s_ties[WAVES];
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
            for (int i = tid; i < budget; i += THREADS) out[i] = !missing && i < len ? i : -1;
        return;
    }

    // slots [first, last) may leave; `want` of them do
    const int first = c.n_sink, last = len - recent, want = len - budget;
    uint32_t prefix = 0, rest = want;              // bits of the want-th lowest score found so far; its place among those that share them
    int shift = 32;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const uint32_t taken = pass == 0 ? 0u : ~0u << shift;            // the bits that prefix has
        shift -= BITS[pass];
        const uint32_t mask = (1u << BITS[pass]) - 1;
        for (int i = tid; i < BINS; i += THREADS) s_hist[i] = 0;
        __syncthreads();
        for (int j = first + tid; j < last; j += THREADS) {
            const uint32_t x = order_of(score[j]);
            if ((x & taken) == prefix) atomicAdd(&s_hist[(x >> shift) & mask], 1u);
        }
        __syncthreads();
        // two bins a thread: running count, and the bin in which it reaches `rest`
        const uint32_t n0 = s_hist[2 * tid], n1 = s_hist[2 * tid + 1];
        uint32_t run = n0 + n1;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t x = __shfl_up(run, d);
            if (lane >= d) run += x;
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
    // Scores below `prefix` leave, and the first `rest` of those equal to it.  A wave takes a stretch of the slots: it counts both,
    // and then knows how many slots stay before it.
    const int stretch = ((len + WAVES - 1) / WAVES + 63) & ~63;
    const int lo = min(len, wave * stretch), hi = min(len, lo + stretch);
    int less = 0, ties = 0;
    for (int j0 = lo; j0 < hi; j0 += 64) {
        const int j = j0 + lane;
        const bool able = j >= first && j < last && j < hi;
        const uint32_t x = able ? order_of(score[j]) : ~0u;
        less += __popcll(__ballot(able && x < prefix));
        ties += __popcll(__ballot(able && x == prefix));
    }
    if (lane == 0) { s_less[wave] = less; s_ties[wave] = ties; }
    __syncthreads();
    int gone = 0, tied = 0;
    for (int w = 0; w < wave; ++w) { gone += s_less[w]; tied += s_ties[w]; }
    int at = lo - gone - min(tied, (int)rest);
    const unsigned long long below = (1ull << lane) - 1;
    for (int j0 = lo; j0 < hi; j0 += 64) {
        const int j = j0 + lane;
        const bool able = j >= first && j < last;
        const uint32_t x = able && j < hi ? order_of(score[j]) : ~0u;
        const bool tie = able && j < hi && x == prefix;
        const unsigned long long tb = __ballot(tie);
        const bool leaves = able && j < hi && (x < prefix || (tie && tied + __popcll(tb & below) < (int)rest));
        const bool stays = j < hi && !leaves;
        const unsigned long long sb = __ballot(stays);
        if (stays) {
            const int i = at + __popcll(sb & below);
            mine[i] = j;
            if (out) out[i] = j;
        }
        at += __popcll(sb);
        tied += __popcll(tb);
    }
}

// What the workgroup has read is there before any of it writes.
__device__ __forceinline__ void read_then_write()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Workgroup x: unit x / (2 * pieces + 1); K's pieces, V's pieces, the sums.
template <int PIECE>
__global__ __launch_bounds__(THREADS)
void wkv_evict_move_kernel(const WkvPages c, int list_stride, int pieces, const int32_t* __restrict__ plan, const int32_t* __restrict__ list,
                           int32_t* __restrict__ new_lens, float* new_scores)
{
    const int unit = blockIdx.x / (2 * pieces + 1), what = blockIdx.x - unit * (2 * pieces + 1);
    const int b = unit / c.kv_heads, h = unit - b * c.kv_heads;
    const int tid = threadIdx.x;
    const int len = plan[2 * b], left = plan[2 * b + 1];
    const int32_t* mine = list + (int64_t)unit * list_stride;
    if (what == 2 * pieces) {
        const float* from = c.scores + (int64_t)unit * c.score_stride;
        float* to = new_scores + (int64_t)unit * c.score_stride;
        if (h == 0 && tid == 0) new_lens[b] = left;
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
    constexpr int LANES = PIECE / 16, ROWS = THREADS / LANES, N = 4;       // rows of a load, loads in flight
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
    constexpr int PIECE = 128;
    const int units = c.batch * c.kv_heads, pieces = row_bytes / PIECE, list_stride = std::min(budget, c.max_slots);
    const int per_unit = 2 * pieces + 1;
    if ((int64_t)units * per_unit >= 1 << 22) return hipErrorInvalidValue;       // 2^32 threads
    hipLaunchKernelGGL(wkv_evict_select_kernel, dim3(units), dim3(THREADS), 0, stream, c, budget, list_stride, recent, kept, plan, list);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((wkv_evict_move_kernel<PIECE>), dim3(units * per_unit), dim3(THREADS), 0, stream, c, list_stride, pieces, plan, list,
                       new_lens, new_scores);
    return hipGetLastError();
}
