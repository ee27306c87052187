// Attention over the paged cache (wkv_paged in include/wkv.h): one new token per sequence, or a chunk of them.
//
// A unit is a sequence and a K/V head.  Its rows are the new tokens times the query heads of the group, row r being token
// r / group and head r % group, so that the heads that share K and V share what is loaded of them.  A tile is 16 rows.
//
//   wkv_paged_rows   a workgroup of four waves takes a tile and a part of the keys that it sees.  Each wave goes over blocks of 32 keys
//                    (16 in fp32 and with wide heads) of its own, from memory straight into registers, with the running maximum and sum of a softmax:
//                    S^T = K Q^T leaves in a lane 4 consecutive keys of one row, which is what the second product's operand
//                    wants (O^T = V^T P^T), so the weights never leave their lane; the values' operand is a transposition of 16-bit
//                    words within a lane.  The waves' sums are joined through LDS.
//   wkv_paged_join   the parts of a row joined (join_few: of few parts, and of many rows).
//                    Behind the joins in the same launch, the weights of a step are summed for every slot, from the logits that
//                    wkv_paged_rows left and the parts' sums (tally).
//   wkv_paged_sums   the weights of a prefill's rows summed for every slot, from the rows' log-sum-exps.
// New K and V rows go into their pages on the way: a call reads its own tokens from where they are, so nothing waits for that.
//
// Softmax statistics, sums of the weights and of weight . v are fp32.
//
// Long steps are bound by memory: 4 x 32768 slots, 32 heads on 8 of 128, fp16: wkv_paged_rows 88.5 us for 537 MB of K and V (6.07 TB/s; 547 MB
// fetched), the join 4.8.  64 ragged sequences of up to 4096 with logits 131 us for 565 + 19 MB, join and tally 13.5.  Short ones by the chain
// launch, table, rows, joins: 4096 slots of one sequence 6.1 + 3.9 us, 64 slots in fp32 4.7.  (Waves that keep K and V in registers, one block
// ahead, and no LDS but for the joins: a first kernel that staged a block at a time took 117 us for the long step, 28 for the one sequence.)
#include "../../include/wkv.h"
#include "wkv_internal.h"
#include "wkv_device.h"
#include "wkv_paged_device.h"

#include <algorithm>
#include <type_traits>

namespace {

constexpr int WAVES = 4, THREADS = 64 * WAVES;

// How a format's rows are cut up for the matrix instructions.
template <class TT, int D> struct Shape {
    static constexpr bool HALF = TT::BYTES == 2;
    // keys of a block: 32, what an instruction of the second product takes; 16 where two blocks of 32 would not fit the
    // registers (that instruction's other half is then zero)
    static constexpr int BK = HALF && D <= 128 ? 32 : 16;
    static constexpr int NT = BK / 16;                     // their tiles of 16
    static constexpr int KL = D * TT::BYTES / 64;          // 16-byte loads of a lane for a key row (four lanes share it)
    static constexpr int VK = BK / 4;                      // keys of a lane's values
    static constexpr int VE = HALF ? (D / 16 < 8 ? D / 16 : 8) : 4;  // consecutive elements of a value row in a lane
    static constexpr int NH = D / (16 * VE);               // such pieces of a row
    static constexpr int VW = VE * TT::BYTES / 4;          // words of a piece
};

// The product over a row (a lane's KL loads): 16-bit rows 8 elements a load and instruction, fp32 rows 4 a load; in fp32 by four sums, whose
// roundings are half of one's.
template <class TT, int KL> __device__ __forceinline__ f32x4_t dot_tile(const u32x4_t (&a)[KL], const u32x4_t (&b)[KL])
{
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    if constexpr (TT::BYTES == 2) {
#pragma unroll
        for (int kk = 0; kk < KL; ++kk) s = mfma<TT>(a[kk], b[kk], s);
    } else {
        f32x4_t t[4] = {};
#pragma unroll
        for (int kk = 0; kk < KL; ++kk) {
            const f32x4_t x = __builtin_bit_cast(f32x4_t, a[kk]), y = __builtin_bit_cast(f32x4_t, b[kk]);
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = mfma_f32(x[e], y[e], t[e]);
        }
        s = (t[0] + t[1]) + (t[2] + t[3]);
    }
    return s;
}

template <class TT, int D> struct Frag {
    using S = Shape<TT, D>;
    u32x4_t k[S::NT][S::KL];
    uint32_t v[S::VK][S::NH][S::VW];
};

// STEP: a row per sequence and head.  EARLY: of a step, where neither a window nor the order of the sequences decides where a wave
// begins.  LOGITS: of a step, whose weights are summed: its logits are stored (with every block, so that waits can be counted).
template <class TT, int D, bool STEP, bool EARLY, bool LOGITS>
__global__ __launch_bounds__(THREADS, D * TT::BYTES > 256 ? 2 : 3)
void wkv_paged_rows_kernel(const WkvPagedCall a)
{
    using S = Shape<TT, D>;
    constexpr int BK = S::BK, NT = S::NT, KL = S::KL, VK = S::VK, VE = S::VE, NH = S::NH, VW = S::VW;
    constexpr int PIECES = D * TT::BYTES / 16;
    __shared__ float s_m[WAVES][ROWS], s_l[WAVES][ROWS];
    __shared__ float s_o[WAVES][ROWS][16 * VE + 4];
    __shared__ u32x4_t s_new[WAVES][2 * PIECES];

    int id = blockIdx.x, tile = 0, unit = 0;
    const bool packed = !STEP && a.slots > 0;
    if (packed) {
        if (!packed_tile(a, id % a.c.kv_heads, id / a.c.kv_heads, unit, tile)) return;
    } else if (a.tiles > 1) {
        // Workgroups are dealt to the chip's eight partitions in turn: the tiles that go over the same keys follow each other on one of them, whose
        // cache then holds those (64 sequences of 8192 slots, 64 heads on one: 156.6 -> 115.5 us).
        if ((int)(gridDim.x / a.tiles) % 8 == 0) {
            const int x = id & 7, y = id >> 3;
            tile = y % a.tiles;
            id = y / a.tiles * 8 + x;
        } else {
            const int per_unit = a.splits * a.tiles, in = id % per_unit;
            tile = in / a.splits;
            id = id / per_unit * a.splits + in % a.splits;
        }
    }
    const int part = packed ? 0 : id % a.splits;
    if (!packed) unit = id / a.splits;
    const WkvPages& c = a.c;
    // Longest sequences first: what is left when the last workgroups have started is short then.
    if (STEP && !EARLY && a.order) {
        __shared__ __attribute__((aligned(16))) int s_len[THREADS];
        __shared__ int s_mine;
        const int place = unit / c.kv_heads, base = place / THREADS * THREADS, n = min(THREADS, c.batch - base);
        const int len = (int)threadIdx.x < n ? max(c.lens[base + threadIdx.x], 0) : -1;       // (places behind the last sequence come last)
        s_len[threadIdx.x] = len;
        __syncthreads();
        int rank = 0;
        for (int i = 0; i < n; i += 4) {
            const int4 x = *reinterpret_cast<const int4*>(&s_len[i]);
            rank += (x.x > len || (x.x == len && i < (int)threadIdx.x)) + (x.y > len || (x.y == len && i + 1 < (int)threadIdx.x)) +
                    (x.z > len || (x.z == len && i + 2 < (int)threadIdx.x)) + (x.w > len || (x.w == len && i + 3 < (int)threadIdx.x));
        }
        if ((int)threadIdx.x < n && rank == place - base) s_mine = base + threadIdx.x;
        __syncthreads();
        unit = __builtin_amdgcn_readfirstlane(s_mine) * c.kv_heads + unit % c.kv_heads;
    }
    const int group = c.group, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    Tile t;
    const bool some = unit_of<STEP>(a, unit, tile * ROWS, t);
    const int r0 = tile * ROWS, r1 = min(t.rows, r0 + ROWS);

    // A step's new rows are taken from where they are, by way of LDS: nothing reads them from their page in this launch.
    const bool append = STEP && a.k_new != nullptr;
    const char* new_k = a.k_new + t.b * a.k_bytes + t.h * a.k_head;
    const char* new_v = a.v_new + t.b * a.v_bytes + t.h * a.v_head;
    if (append && lane < 2 * PIECES)
        s_new[wave][lane] = reinterpret_cast<const u32x4_t*>(lane < PIECES ? new_k : new_v)[lane < PIECES ? lane : lane - PIECES];

    // the lane's row: its query as the second operand of K Q^T
    const int row = r0 + col, row_q = min(row, max(r1, 1) - 1);
    const int token = STEP ? 0 : row_q / group;
    u32x4_t q[KL];
    if (some) {
        const char* src = a.q + (t.q.row0 + token) * a.q_bytes + (t.h * group + row_q - token * group) * a.q_head + g * 16;
#pragma unroll
        for (int kk = 0; kk < KL; ++kk) q[kk] = *reinterpret_cast<const u32x4_t*>(src + kk * 64);
    }

    const int in_page = (1 << c.page_shift) - 1;
    // page of the tile of 16 slots from `pos` on, as the table says, and -1 for what is none
    const int32_t* table = c.table + t.b * c.table_stride;
    auto entry = [&](int pos) { return load_uniform(table + min(pos >> c.page_shift, c.max_pages - 1)); };
    auto page_of = [&](int pos, int page) { return (unsigned)page < (unsigned)c.n_pages && pos < c.max_slots ? page : -1; };

    const char* kh = c.k + t.h * c.head_bytes;
    const char* vh = c.v + t.h * c.head_bytes;
    const uint32_t k_off = (uint32_t)(col * (int)c.slot_bytes) + g * 16;
    const uint32_t v_off = (uint32_t)(g * 4 * (int)c.slot_bytes) + col * (VE * TT::BYTES);
    // A chunk's own tokens, from slot `fresh` on, are read from where they are.  Pages that are not there are loaded as page 0 (it is in the
    // pool) and masked.
    const int fresh = !STEP && a.k_new ? t.pos0 : 0x7FFFFFFF;
    const char* kf = a.k_new + t.h * a.k_head + (t.q.row0 - t.pos0) * a.k_bytes;
    const char* vf = a.v_new + t.h * a.v_head + (t.q.row0 - t.pos0) * a.v_bytes;
    Frag<TT, D> x;
    auto row0 = [&](int pos, int page) { return max(page, 0) * c.page_bytes + (pos & in_page) * c.slot_bytes; };
    auto load_k = [&](int pos, const int (&pages)[NT]) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int kk = 0; kk < KL; ++kk) {
                const char* src = kh + row0(pos + i * 16, pages[i]) + k_off;
                if (!STEP && pos + i * 16 + col >= fresh && pos + i * 16 + col < t.q.len) src = kf + (pos + i * 16 + col) * a.k_bytes + g * 16;
                x.k[i][kk] = *reinterpret_cast<const u32x4_t*>(src + kk * 64);
            }
    };
    // (A step reads every row once, and its V rows whole by every load: non-temporal.  K rows, a half line by every load, are better off without:
    // 4 x 32768 slots 96 -> 100 us, 64 ragged sequences 154 -> 177.)
    auto load_v = [&](int pos, const int (&pages)[NT]) {
#pragma unroll
        for (int j = 0; j < VK; ++j)
#pragma unroll
            for (int h = 0; h < NH; ++h) {
                const int p = pos + j / 4 * 16 + g * 4 + j % 4;
                const char* src = vh + (row0(pos + j / 4 * 16, pages[j / 4]) + j % 4 * c.slot_bytes) + v_off;
                if (!STEP && p >= fresh && p < t.q.len) src = vf + p * a.v_bytes + col * (VE * TT::BYTES);
                load_words<VW, STEP>(src + h * (16 * VE * TT::BYTES), x.v[j][h]);
            }
    };

    // The blocks go to the parts' waves in turn: where a wave begins does not depend on the length (but under a window), so its first
    // block is on its way when the length is not known yet.  From there on a block's K rows are requested when those before them have been
    // used, and its V rows likewise: each has the other's part of the work to arrive in, and takes the registers of the ones before.
    // Behind the last block that one is loaded again (a load that is there on every path is what the waits are counted by).
    int pos[3] = {0, 0, 0}, pages[3][NT];          // of the block in use, the one that travels, the one after it
    auto known = [&](int p, int (&e)[NT]) {
#pragma unroll
        for (int i = 0; i < NT; ++i) e[i] = page_of(p + i * 16, e[i]);
    };
    const int mine = part * WAVES + wave, stride = a.splits * WAVES;
    if constexpr (EARLY) {
        pos[0] = mine * BK;
#pragma unroll
        for (int i = 0; i < NT; ++i) pages[0][i] = entry(pos[0] + i * 16);
        known(pos[0], pages[0]);
        load_k(pos[0], pages[0]);
        load_v(pos[0], pages[0]);
    }

    if (!some) return;
    const int p_lo = STEP ? t.pos0 : t.pos0 + r0 / group, p_hi = STEP ? t.pos0 : t.pos0 + (r1 - 1) / group;
    const int window = !EARLY && c.window > 0 ? c.window : 0x40000000;
    const Span sp = span(a, p_lo, p_hi);
    if (part >= sp.parts) return;
    const bool row_ok = row < r1;
    const int p_row = STEP ? t.pos0 : row_ok ? t.pos0 + token : -1;          // (a step's lanes without a row have the last one's)
    const int pos_new = append ? p_lo : -1;
    if (append && part == 0 && tile == 0 && wave == WAVES - 1 && pos_new >= 0) {
        const int page = page_of(pos_new, entry(pos_new));
        if (page >= 0 && lane < 2 * PIECES) {
            char* to = (lane < PIECES ? c.k : c.v) + page * c.page_bytes + (pos_new & in_page) * c.slot_bytes + t.h * c.head_bytes;
            *reinterpret_cast<u32x4_t*>(to + (lane < PIECES ? lane : lane - PIECES) * 16) = s_new[wave][lane];
        }
    }
    if (!STEP && a.k_new && part == 0)
        append_rows<D * TT::BYTES, THREADS>(a, t, (r0 + group - 1) / group, min(t.q.n, (r0 + ROWS + group - 1) / group));
    auto slot_of = [&](int blk) { const int i = blk * BK; return EARLY || i < sp.first ? i : i - sp.first + sp.lo; };
    const int count = mine < sp.blocks ? (sp.blocks - mine + stride - 1) / stride : 0;
    auto ahead = [&](int k, int& p, int (&e)[NT]) {
        p = __builtin_amdgcn_readfirstlane(slot_of(mine + stride * min(k, count - 1)));
#pragma unroll
        for (int i = 0; i < NT; ++i) e[i] = entry(p + i * 16);
    };
    auto shift = [&] {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            pos[x] = pos[x + 1];
#pragma unroll
            for (int i = 0; i < NT; ++i) pages[x][i] = pages[x + 1][i];
        }
    };

    float m = -INFINITY, l = 0.f;
    f32x4_t o[NH][VE];
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int e = 0; e < VE; ++e) o[h][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    constexpr float RAISED = __is_same(TT, TF16) ? 0x1p15f : 1.f;          // what the weights are multiplied by, as operands, and so the sums
    auto scale_all = [&](float f) {
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int e = 0; e < VE; ++e) o[h][e] *= f;
    };

    // one block, and the loads of the next one
    auto use = [&](int pos, const int (&pages)[NT], int next, const int (&next_pages)[NT]) {
        const bool fresh = STEP && (unsigned)(pos_new - pos) < (unsigned)BK;
        if (fresh) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
                if (col == pos_new - pos - i * 16)
#pragma unroll
                    for (int kk = 0; kk < KL; ++kk) x.k[i][kk] = s_new[wave][g + kk * 4];
        }
        f32x4_t s[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) s[i] = dot_tile<TT, KL>(x.k[i], q);
        load_k(next, next_pages);
        bool there = true;
#pragma unroll
        for (int i = 0; i < NT; ++i) there &= pages[i] >= 0;
        // every row of the tile sees every key of the block
        const bool full = there && pos + BK - 1 <= p_lo && (pos > p_hi - window || pos + BK <= c.n_sink);
        if (!full) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int p = pos + i * 16 + g * 4 + j;
                    const bool seen = pages[i] >= 0 && p <= p_row && (p > p_row - window || p < c.n_sink);
                    s[i][j] = seen ? s[i][j] : -INFINITY;
                }
        }
        float low = INFINITY;                             // the lowest logit that is seen
        if constexpr (RAISED != 1.f) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) low = fminf(low, full ? s[i][j] : s[i][j] == -INFINITY ? INFINITY : s[i][j]);
        }
        if constexpr (LOGITS) {
            float* dst = a.logits + ((int64_t)unit * group + row_q) * a.logit_stride + pos + g * 4;
#pragma unroll
            for (int i = 0; i < NT; ++i) *reinterpret_cast<f32x4_t*>(dst + i * 16) = s[i];
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, s[i][j] * a.scale);
        {
            float x0, x1;
            lane_pair<16>(top, x0, x1); top = fmaxf(x0, x1);
            lane_pair<32>(top, x0, x1); top = fmaxf(x0, x1);
        }
        if (__any(top > m)) {
            const float f0 = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top);
            m = top;
            l *= f0;
            scale_all(f0);
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float p[NT][4];
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[i][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][j], a.scale, -ref));
                l += p[i][j];
            }
        if (fresh) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (g * 4 + j == pos_new - pos - i * 16)
#pragma unroll
                        for (int h = 0; h < NH; ++h)
#pragma unroll
                            for (int w = 0; w < VW; ++w)
                                x.v[i * 4 + j][h][w] = reinterpret_cast<const uint32_t*>(&s_new[wave][PIECES])[(h * 16 + col) * VW + w];
        }
        if (!full) {
            // values that no row sees have no effect, whatever they are
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int p = pos + i * 16 + g * 4 + j;
                    const bool any = pages[i] >= 0 && p <= p_hi && (p > p_lo - window || p < c.n_sink);
#pragma unroll
                    for (int h = 0; h < NH; ++h)
#pragma unroll
                        for (int w = 0; w < VW; ++w) {
                            uint32_t& word = x.v[i * 4 + j][h][w];
                            word = any ? word : 0u;
                        }
                }
        }
        if constexpr (S::HALF) {
            // element e of the lane's keys
            auto values = [&](int h, int e) {
                u32x4_t vt = {};
#pragma unroll
                for (int w = 0; w < VK / 2; ++w)
                    vt[w] = __builtin_amdgcn_perm(x.v[2 * w + 1][h][e / 2], x.v[2 * w][h][e / 2], (e & 1) ? 0x07060302u : 0x05040100u);
                return vt;
            };
            if constexpr (RAISED != 1.f) {
                // fp16 has no numbers below 2^-24, so weights are raised by 2^15, up to what it can hold, and those that are still below 2^-9, where the
                // second number has no bits left, go by themselves, raised by 2^24 more: 2^-16 of a weight down to 2^-48 of a row's largest, and
                // 2^-64 of that one below.  (A key that takes nearly all of a row with a value near 0 leaves the output to such weights.)
                constexpr float SMALL = 0x1p-9f, MORE = 0x1p24f;
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) p[i][j] *= RAISED;
                asm volatile("" : "+v"(l));
                if (__builtin_expect(__any(__builtin_fmaf(low, a.scale, -ref) < -24.f), 0)) {                // (2^-9, raised)
                    scale_all(MORE);
#pragma unroll 1
                    for (int second = 0; second < 2; ++second) {              // (one number at a time: registers are scarce)
                        u32x4_t part = {};
#pragma unroll
                        for (int w = 0; w < VK / 2; ++w) {
                            float x0 = p[w >> 1][(w & 1) * 2], x1 = p[w >> 1][(w & 1) * 2 + 1];
                            x0 = x0 < SMALL ? x0 * MORE : 0.f;
                            x1 = x1 < SMALL ? x1 * MORE : 0.f;
                            part[w] = pack2<TT>(x0, x1);
                            if (second) {
                                float y0, y1;
                                unpack2<TT>(part[w], y0, y1);
                                part[w] = pack2<TT>(x0 - y0, x1 - y1);
                            }
                        }
#pragma unroll
                        for (int h = 0; h < NH; ++h)
#pragma unroll
                            for (int e = 0; e < VE; ++e) {
                                o[h][e] = mfma<TT>(values(h, e), part, o[h][e]);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                        // (what this makes of the values is not kept in registers)
#pragma unroll
                        for (int j = 0; j < VK; ++j)
#pragma unroll
                            for (int h = 0; h < NH; ++h)
#pragma unroll
                                for (int w = 0; w < VW; ++w) asm volatile("" : "+v"(x.v[j][h][w]));
                    }
                    scale_all(1.f / MORE);
#pragma unroll
                    for (int i = 0; i < NT; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) p[i][j] = p[i][j] < SMALL ? 0.f : p[i][j];
                }
            }
            // The weights as a sum of two 16-bit numbers: what is left of them is below 2^-16 of a weight.  One number
            // alone would err as much as the rounding of the output.
            u32x4_t hi = {}, lo = {};
#pragma unroll
            for (int w = 0; w < VK / 2; ++w) {
                const float x0 = p[w >> 1][(w & 1) * 2], x1 = p[w >> 1][(w & 1) * 2 + 1];
                hi[w] = pack2<TT>(x0, x1);
                float y0, y1;
                unpack2<TT>(hi[w], y0, y1);
                lo[w] = pack2<TT>(x0 - y0, x1 - y1);
            }
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const u32x4_t vt = values(h, e);
                    o[h][e] = mfma<TT>(vt, hi, o[h][e]);
                    o[h][e] = mfma<TT>(vt, lo, o[h][e]);
                }
        } else {
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int e = 0; e < VE; ++e)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[h][e] = mfma_f32(__builtin_bit_cast(float, x.v[j][h][e]), p[0][j], o[h][e]);
        }
        load_v(next, next_pages);
    };

    if (count > 0) {
        if constexpr (!EARLY) {
            ahead(0, pos[0], pages[0]);
            known(pos[0], pages[0]);
            load_k(pos[0], pages[0]);
            load_v(pos[0], pages[0]);
        }
        ahead(1, pos[1], pages[1]);
        for (int k = 0; k < count; ++k) {
            known(pos[1], pages[1]);
            ahead(k + 2, pos[2], pages[2]);
            use(pos[0], pages[0], pos[1], pages[1]);
            shift();
        }
    }

    // A value that is not finite spoils the matrix product: it meets weights of 0 of rows that do not see it, and parts of weights that are 0
    // or negative; and sums of the largest values may overflow.  If one is not finite, the wave forms its sums anew, key by key: a lane has a row
    // and a quarter of the elements.
    {
        float z = 0.f;
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int e = 0; e < VE; ++e)
#pragma unroll
                for (int r = 0; r < 4; ++r) z = __builtin_fmaf(o[h][e][r], 0.f, z);
        if (__any(z != 0.f)) {                            // (0 x infinity and 0 x NaN are NaN, which is no 0)
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int e = 0; e < VE; ++e) o[h][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            const char* qr = a.q + (t.q.row0 + token) * a.q_bytes + (t.h * group + row_q - token * group) * a.q_head;
            m += CAREFUL<TT>;
            l *= __builtin_amdgcn_exp2f(-CAREFUL<TT>);
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll 1
            for (int i = 0; i < count * BK; ++i) {
                const int p = slot_of(mine + stride * (i / BK)) + i % BK;
                const int page = page_of(p, entry(p));
                if (page < 0) continue;
                const int64_t at = page * c.page_bytes + (p & in_page) * c.slot_bytes;
                if (p >= t.q.len) continue;
                const char* kr = p == pos_new ? new_k : p >= fresh ? kf + p * a.k_bytes : kh + at;
                const char* vr = p == pos_new ? new_v : p >= fresh ? vf + p * a.v_bytes : vh + at;
                float dot = 0.f;
#pragma unroll 1
                for (int e = g * (D / 4); e < (g + 1) * (D / 4); ++e) dot += load_elem<TT>(qr, e) * load_elem<TT>(kr, e);
                dot = rows_sum(dot);
                if (p <= p_row && (p > p_row - window || p < c.n_sink)) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(dot, a.scale, -ref)) * RAISED;
#pragma unroll
                    for (int h = 0; h < NH; ++h)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int e = 0; e < VE; ++e) o[h][e][r] += w * load_elem<TT>(vr, h * 16 * VE + (g * 4 + r) * VE + e);
                }
            }
        }
    }

    // ---- the four waves' sums joined
    l = rows_sum(l);
    if (g == 0) { s_m[wave][col] = m; s_l[wave][col] = l; }
    __syncthreads();
    float top = s_m[0][col];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, s_m[w][col]);
    top += JOINED;
    const float share = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    const bool direct = sp.parts == 1;
    int tid = threadIdx.x;
    asm("" : "+v"(tid));                                  // (not kept in registers through the loop above)
    const int orow = tid >> 4, piece = tid & 15;                           // 16 lanes write a row
    const bool own = r0 + orow < r1;
    float sum = 0.f, otop = s_m[0][orow];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) otop = fmaxf(otop, s_m[w][orow]);
    otop += JOINED;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += s_m[w][orow] == -INFINITY ? s_l[w][orow] : s_l[w][orow] * __builtin_amdgcn_exp2f(s_m[w][orow] - otop);
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    const int64_t cell = ((int64_t)unit * a.tiles + tile) * a.splits + part;
    const int otoken = STEP ? 0 : min(r0 + orow, r1 - 1) / group, ohead = t.h * group + min(r0 + orow, r1 - 1) - otoken * group;
    char* dst = a.out + (t.q.row0 + otoken) * a.out_bytes + ohead * a.out_head;
#pragma unroll
    for (int h = 0; h < NH; ++h) {
        if (h > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < VE; ++e) s_o[wave][col][(g * 4 + r) * VE + e] = o[h][e][r] * (share * (1.f / RAISED));
        __syncthreads();
        float x[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            x[e] = s_o[0][orow][piece * VE + e];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) x[e] += s_o[w][orow][piece * VE + e];
        }
        if (!own) continue;
        if (direct) {
            uint32_t w[VW];
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                if constexpr (S::HALF) w[e] = pack2<TT>(mean<TT>(x[2 * e], inv), mean<TT>(x[2 * e + 1], inv));
                else w[e] = __builtin_bit_cast(uint32_t, mean<TT>(x[e], inv));
            }
            store_words<VW>(dst + (h * 16 + piece) * (VE * TT::BYTES), w);
        } else {
            float* p = a.part + (cell * ROWS + orow) * D + (h * 16 + piece) * VE;
#pragma unroll
            for (int e = 0; e < VE; e += 4) *reinterpret_cast<f32x4_t*>(p + e) = f32x4_t{x[e], x[e + 1], x[e + 2], x[e + 3]};
        }
    }
    if (piece == 0 && own) {
        if (a.ml) { a.ml[cell * 32 + orow] = otop; a.ml[cell * 32 + 16 + orow] = sum; }
        if (!STEP && a.lse && direct)
            a.lse[(int64_t)(t.q.row0 + otoken) * (c.kv_heads * group) + ohead] = otop == -INFINITY ? INFINITY : otop + __builtin_amdgcn_logf(sum);
    }
}

// ---------------------------------------------------------------- joining
constexpr int TALLY = 512;           // slots whose weights one workgroup sums

// What a row's parts come to: their largest reference and the sum of the weights by it, in all lanes; the lane's part's share.  (Of at
// most 64 parts, one to a lane.)
__device__ __forceinline__ void parts_of(const float* ml, int parts, int most, int lane, float& top, float& sum, float& share)
{
    // (cells of parts that there are not are in the workspace too: loading them waits for nothing)
    float m = -INFINITY, l = 0.f;
    if (lane < most) { m = ml[lane * 32]; l = ml[lane * 32 + 16]; }
    if (lane >= parts) { m = -INFINITY; l = 0.f; }
    top = m;
    top = fmaxf(top, dpp<0xB1>(top)); top = fmaxf(top, dpp<0x4E>(top)); top = fmaxf(top, dpp<0x141>(top)); top = fmaxf(top, dpp<0x140>(top));
    float x0, x1;
    lane_pair<16>(top, x0, x1); top = fmaxf(x0, x1);
    lane_pair<32>(top, x0, x1); top = fmaxf(x0, x1) + JOINED;
    share = m == -INFINITY ? (l == l ? 0.f : l) : __builtin_amdgcn_exp2f(m - top);
    sum = rows_sum(row_allsum(m == -INFINITY ? l : l * share));
}

// Weights of a step, summed over a unit's heads and added to the slots' sums: a workgroup takes TALLY of the keys that the unit saw,
// in the order of span().
constexpr int HEADS = 256;           // heads of a unit whose log-sum-exps are at hand at a time
__device__ __forceinline__ void tally(const WkvPagedCall& a, int block, int per_unit)
{
    __shared__ float s_lse[HEADS];
    const int unit = block / per_unit, first = block % per_unit * TALLY;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = a.c.group;
    Tile t;
    unit_of<true>(a, unit, 0, t);
    const Span sp = span(a, t.pos0, t.pos0);
    const int keys = t.pos0 < 0 ? 0 : sp.first + t.pos0 + 1 - sp.lo;
    if (first >= keys) return;
    constexpr int N = TALLY / THREADS;
    float w[N] = {};
    int at[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = min(first + i * THREADS + (int)threadIdx.x, keys - 1);
        at[i] = j < sp.first ? j : j - sp.first + sp.lo;
    }
    for (int g0 = 0; g0 < group; g0 += HEADS) {
        const int n = min(HEADS, group - g0);
        for (int r = wave; r < n; r += WAVES) {
            float top, sum, share;
            parts_of(a.ml + ((int64_t)unit * a.tiles + (g0 + r) / ROWS) * a.splits * 32 + (g0 + r) % ROWS, sp.parts, a.splits, lane, top, sum, share);
            if (lane == 0) s_lse[r] = top == -INFINITY ? INFINITY : top + __builtin_amdgcn_logf(sum);
        }
        __syncthreads();
        const float* lg = a.logits + ((int64_t)unit * group + g0) * a.logit_stride;
#pragma unroll 4
        for (int r = 0; r < n; ++r)
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(lg[r * a.logit_stride + at[i]], a.scale, -s_lse[r]));
        __syncthreads();
    }
    float* sc = a.c.scores + (int64_t)unit * a.c.score_stride;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (first + i * THREADS + (int)threadIdx.x >= keys) continue;
        if (w[i] != w[i]) {
            // some row has no finite weights, which gives it none on what it does not see either: a missing page, or what lies beside the window in its blocks
            const int page = a.c.table[t.b * a.c.table_stride + (at[i] >> a.c.page_shift)];
            const bool seen = (unsigned)page < (unsigned)a.c.n_pages && (a.c.window <= 0 || at[i] > t.pos0 - a.c.window || at[i] < a.c.n_sink);
            w[i] = seen ? w[i] : 0.f;
        }
        if (at[i] == t.pos0 && a.k_new) sc[at[i]] = w[i];
        else sc[at[i]] += w[i];
    }
}

// The joined row's output, and its log-sum-exp for a prefill whose weights are summed.
template <class TT, bool STEP>
__device__ __forceinline__ void put_row(const WkvPagedCall& a, const Tile& t, int row, int x4, f32x4_t y, float top, float sum)
{
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    const int token = STEP ? 0 : row / a.c.group, head = t.h * a.c.group + row - token * a.c.group;
    char* dst = a.out + (t.q.row0 + token) * a.out_bytes + head * a.out_head + x4 * (4 * TT::BYTES);
    if constexpr (TT::BYTES == 2)
        *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<TT>(mean<TT>(y[0], inv), mean<TT>(y[1], inv)), pack2<TT>(mean<TT>(y[2], inv), mean<TT>(y[3], inv)));
    else
        *reinterpret_cast<f32x4_t*>(dst) = f32x4_t{mean<TT>(y[0], inv), mean<TT>(y[1], inv), mean<TT>(y[2], inv), mean<TT>(y[3], inv)};
    if (!STEP && a.lse && x4 == 0)
        a.lse[(int64_t)(t.q.row0 + token) * (a.c.kv_heads * a.c.group) + head] = top == -INFINITY ? INFINITY : top + __builtin_amdgcn_logf(sum);
}

template <bool STEP> __device__ __forceinline__ Span span_of_row(const WkvPagedCall& a, const Tile& t, int row)
{
    if constexpr (STEP) return span(a, t.pos0, t.pos0);
    const int t0 = row & -a.tile_rows, t1 = min(t.rows, t0 + a.tile_rows);          // (the keys were cut into parts for that tile)
    return span(a, t.pos0 + t0 / a.c.group, t.pos0 + (t1 - 1) / a.c.group);
}

// Workgroups 0 .. joins - 1 join the parts of rows; behind them, for a step whose weights are summed, they tally.
//
// Row x of all cells (per_tile of each): a workgroup joins SETS rows of a few parts, D / 4 lanes each.
constexpr int FEW = 4, SOME = 16, MANY = 1024;
template <class TT, int D, int MOST, bool STEP>
__global__ __launch_bounds__(THREADS)
void wkv_paged_join_few_kernel(const WkvPagedCall a, int joins, int rows, int per_tile, int per_unit)
{
    if constexpr (STEP) {
        if ((int)blockIdx.x >= joins) return tally(a, blockIdx.x - joins, per_unit);
    }
    constexpr int LANES = D / 4, SETS = THREADS / LANES;
    const int x = blockIdx.x * SETS + threadIdx.x / LANES, x4 = threadIdx.x % LANES;
    if (x >= rows) return;
    const int at = x % per_tile, cell = x / per_tile, unit = cell / a.tiles, row = (cell - unit * a.tiles) * ROWS + at;
    Tile t;
    if (!unit_of<STEP>(a, unit, row, t)) return;
    const Span sp = span_of_row<STEP>(a, t, row);
    if (sp.parts == 1) return;
    const float* ml = a.ml + (int64_t)cell * a.splits * 32 + at;
    const float* src = a.part + ((int64_t)cell * a.splits * ROWS + at) * D + x4 * 4;
    float m[MOST], l[MOST], top = -INFINITY, sum = 0.f;
    f32x4_t v[MOST], y = {0.f, 0.f, 0.f, 0.f};
    // (in place of parts that there are not the last one is loaded: no branch between the loads)
#pragma unroll
    for (int i = 0; i < MOST; ++i)
        if (i < a.splits) {
            const int part = min(i, sp.parts - 1);
            m[i] = ml[part * 32];
            l[i] = ml[part * 32 + 16];
            v[i] = *reinterpret_cast<const f32x4_t*>(src + (int64_t)part * ROWS * D);
        }
#pragma unroll
    for (int i = 0; i < MOST; ++i) if (i < a.splits) top = fmaxf(top, m[i]);
    top += JOINED;
#pragma unroll
    for (int i = 0; i < MOST; ++i)
        if (i < sp.parts) {
            const float f = m[i] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - top);
            sum += f * l[i];
            y += f * v[i];
        }
    put_row<TT, STEP>(a, t, row, x4, y, top, sum);
}

// The same for up to 64 parts, a workgroup a row: its waves' lanes sum parts side by side.
template <class TT, int D, bool STEP>
__global__ __launch_bounds__(THREADS, 4)
void wkv_paged_join_kernel(const WkvPagedCall a, int joins, int per_tile, int per_unit)
{
    if constexpr (STEP) {
        if ((int)blockIdx.x >= joins) return tally(a, blockIdx.x - joins, per_unit);
    }
    constexpr int LANES = D / 4, SETS = THREADS / LANES, DEEP = 64 / SETS;         // parts side by side, one after the other
    __shared__ f32x4_t s_x[SETS][LANES];
    const int lane = threadIdx.x & 63;
    const int at = blockIdx.x % per_tile, cell = blockIdx.x / per_tile, unit = cell / a.tiles, row = (cell - unit * a.tiles) * ROWS + at;
    const float* ml = a.ml + (int64_t)cell * a.splits * 32 + at;
    const int set = threadIdx.x / LANES, x4 = threadIdx.x % LANES;
    const float* src = a.part + ((int64_t)cell * a.splits * ROWS + at) * D + x4 * 4;
    f32x4_t x[DEEP];
#pragma unroll
    for (int i = 0; i < DEEP; ++i)
        if (i * SETS + set < a.splits) x[i] = *reinterpret_cast<const f32x4_t*>(src + (int64_t)(i * SETS + set) * ROWS * D);
    Tile t;
    if (!unit_of<STEP>(a, unit, row, t)) return;
    const Span sp = span_of_row<STEP>(a, t, row);
    if (sp.parts == 1) return;
    float top, sum, share;
    parts_of(ml, sp.parts, a.splits, lane, top, sum, share);
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < DEEP; ++i) {
        const float f = __shfl(share, i * SETS + set);
        if (i * SETS + set < sp.parts) y += f * x[i];
    }
    s_x[set][x4] = y;
    __syncthreads();
    if (set > 0) return;
#pragma unroll
    for (int i = 1; i < SETS; ++i) y += s_x[i][x4];
    put_row<TT, STEP>(a, t, row, x4, y, top, sum);
}

// ---------------------------------------------------------------- weights of a prefill's rows, summed for every slot
constexpr int SUM_KEYS = 64;         // keys of a wave

// S = Q K^T with the keys' operands in registers: a lane has four rows of one key, so the sum over rows is within the lane but for
// the last step.  A wave goes over all tiles of rows that see its keys.
template <class TT, int D>
__global__ __launch_bounds__(THREADS, 2)
void wkv_paged_sums_kernel(const WkvPagedCall a, int unit0, int per_unit)
{
    using S = Shape<TT, D>;
    constexpr int KL = S::KL, KT = D * TT::BYTES > 256 ? 2 : 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const WkvPages& c = a.c;
    const int unit = unit0 + blockIdx.x / per_unit;
    Tile t;
    if (!unit_of<false>(a, unit, 0, t)) return;
    const int window = c.window > 0 ? c.window : 0x40000000, group = c.group;
    const int in_page = (1 << c.page_shift) - 1;
#pragma unroll 1
    for (int sub = 0; sub < 4 / KT; ++sub) {
        const int k0 = ((blockIdx.x % per_unit) * WAVES + wave) * SUM_KEYS + sub * KT * 16;
        if (k0 >= t.q.len) return;
        u32x4_t k[KT][KL];
        bool there[KT];
#pragma unroll
        for (int i = 0; i < KT; ++i) {
            const int p = k0 + i * 16, n = p >> c.page_shift;
            const int page = n < c.max_pages ? c.table[t.b * c.table_stride + n] : -1;
            there[i] = (unsigned)page < (unsigned)c.n_pages;
            const char* src = c.k + (there[i] ? page : 0) * c.page_bytes + ((p + col) & in_page) * c.slot_bytes + t.h * c.head_bytes + g * 16;
#pragma unroll
            for (int kk = 0; kk < KL; ++kk) k[i][kk] = *reinterpret_cast<const u32x4_t*>(src + kk * 64);
        }
        // tokens that see some key of these
        const int i0 = max(0, k0 - t.pos0);
        const bool sinks = k0 < c.n_sink;
        const int i1 = sinks ? t.q.n : (int)min((int64_t)t.q.n, (int64_t)k0 + KT * 16 - 1 + window - t.pos0);
        float sum[KT] = {};
        for (int r0 = i0 * group & ~15; r0 < i1 * group; r0 += ROWS) {
            const int row = min(r0 + col, t.rows - 1);
            const int token = row / group, head = t.h * group + row - token * group;
            const char* src = a.q + (t.q.row0 + token) * a.q_bytes + head * a.q_head + g * 16;
            u32x4_t q[KL];
#pragma unroll
            for (int kk = 0; kk < KL; ++kk) q[kk] = *reinterpret_cast<const u32x4_t*>(src + kk * 64);
            float lse[4];
            int pr[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = min(r0 + g * 4 + j, t.rows - 1), tk = r / group, hd = t.h * group + r - tk * group;
                lse[j] = a.lse[(int64_t)(t.q.row0 + tk) * (c.kv_heads * group) + hd];
                pr[j] = r0 + g * 4 + j < t.rows ? t.pos0 + tk : -1;
            }
#pragma unroll
            for (int i = 0; i < KT; ++i) {
                const f32x4_t s = dot_tile<TT, KL>(q, k[i]);
                const int p = k0 + i * 16 + col;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j], a.scale, -lse[j]));
                    sum[i] += p <= pr[j] && (p > pr[j] - window || p < c.n_sink) ? w : 0.f;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < KT; ++i) {
            const float x = rows_sum(sum[i]);
            const int p = k0 + i * 16 + col;
            if (g == 0 && p < t.q.len) {
                float* sc = c.scores + (int64_t)unit * c.score_stride + p;
                const float w = there[i] ? x : 0.f;
                if (a.k_new && p >= t.pos0) *sc = w;
                else if (there[i]) *sc += w;
            }
        }
    }
}

template <class F> hipError_t by_type(int dtype, int head_dim, F&& f)
{
    if (dtype == WKV_FP32) return head_dim == 64 ? f(TF32{}, std::integral_constant<int, 64>{}) : f(TF32{}, std::integral_constant<int, 128>{});
    auto wide = [&](auto t) {
        return head_dim == 64 ? f(t, std::integral_constant<int, 64>{}) : head_dim == 128 ? f(t, std::integral_constant<int, 128>{})
                                                                                          : f(t, std::integral_constant<int, 256>{});
    };
    return dtype == WKV_FP16 ? wide(TF16{}) : wide(TBF16{});
}

}  // namespace

int64_t wkv_paged_most_keys(const WkvPages& c, int64_t new_tokens)
{
    return c.window > 0 ? std::min<int64_t>(c.max_slots, (int64_t)c.window + c.n_sink + new_tokens + 128) : c.max_slots;
}

void wkv_paged_shape(WkvPagedCall& a, int64_t units, int64_t rows, int64_t most, int dtype, int head_dim, bool step)
{
    a.tiles = (int)((rows + ROWS - 1) / ROWS);
    // The kernel for many rows is ahead from about 32 rows on (2000 slots: 20 rows 19.4 us against 15.6 of the other, 48 rows 19.4 | 20.0; 80 rows onto 8000
    // slots 23 | 43), but not for short prompts that leave the chip half empty either way (77 tokens of 32 K/V heads 15.2 | 12.5, 256 tokens of 8 with
    // four query heads each 17.9 | 16.0; 4 x 128 of these 15.8 | 20.7).  Steps, of however many heads, are the other's: it has their rows without `starts`
    // and keeps their logits.
    a.many = !step && dtype != WKV_FP32 && rows > 32 && (units * a.tiles > 512 || a.c.max_slots > 256);
    a.tile_rows = a.many ? 128 : ROWS;
    const int64_t groups = units * ((rows + a.tile_rows - 1) / a.tile_rows);
    auto over = [&](int64_t n) { return (n + groups - 1) / groups; };
    auto parts = [&](int64_t want, int64_t least) { return (int)std::max<int64_t>(1, std::min<int64_t>({want, (most + least - 1) / least, 64})); };
    // Chunks of different lengths: room for the tiles that n_tokens can have, where as many as the longest chunk has for every sequence are several times
    // that.  us with a workgroup for each of these | packed: 64 chunks of 128 tokens and one of 512 (3 times) 136 | 138, of 128 and 1024 (6) 148 | 155,
    // 200 of 64 and 1024 (10) 109 | 100, 64 of 64 and 2048 (16) 165 | 139, 256 of 4 and 8192 (121) 1104 | 670; the other kernel, fp32, 128 of 64 and 512
    // (3) 104 | 84, of 16 and 1024 (7) 132 | 56.
    a.slots = 0;
    auto pack = [&] {
        if (step || a.splits > 1) return;
        const int64_t slots = (int64_t)a.n_tokens * a.c.group / a.tile_rows + a.c.batch;
        if (groups > (a.many ? 8 : 2) * slots * a.c.kv_heads) a.slots = (int)slots;
    };
    if (a.many) {
        // Parts of 384 keys at least, as many as three workgroups a compute unit want; two for a prompt, whose tiles are of different lengths anyway.
        // us with 256 | 512 | 768 workgroups wanted: 3 x 333 tokens on 6001 190 | 159 | 171, of ragged lengths 185 | 120 | 99, 2 x 500 on 16000 489 | 359 | 336,
        // 100 on 32000 140 | 106 | 101, 1000 on 8000 255 | 172 | 161, 1300 55 | 51 | 53, 2 x 3000 of 512 bytes 234 | 232 | 271.
        a.splits = parts(over((int64_t)a.max_new * 2 > a.c.max_slots ? 512 : 768), 384);
        a.block = head_dim == 64 || (head_dim == 128 && groups * a.splits <= 512) ? 64 : 32;
        a.least = 384 / a.block;
        pack();
        return;
    }
    a.block = dtype == WKV_FP32 || head_dim > 128 ? 16 : 32;
    a.least = WAVES;
    // A workgroup for each of the 256 compute units, or, where parts stay as long as 1024 keys, three, which run side by side (two with wide
    // rows).  More and shorter parts cost more at their ends than they gain.  us a step with 256 | 512 | 768 | 1024 workgroups wanted:
    // 16 sequences of 2047 slots, 2 K/V heads for 32 heads 14.5 | 16.8 | 16.8 | 18.6, the same with rows of 512 bytes 20.8 | 22.9 | 29.5 | 32.5,
    // 1 x 4096, 32 K/V heads 19.1 | 21.5 | 21.9 | 23.9, 8 x 8192 48.8 | 50.8 | 48.6 | 55.7, 4 x 32768 95.8 | 98.0 | 92.7.
    a.splits = parts(std::max(over(256), std::min(over(768), most / 1024)), (int64_t)a.block * a.least);
    // More workgroups than run at once: the longest sequences first (64 ragged sequences, 1024 workgroups: 157 -> 148 us).
    a.order = step && a.c.batch > 1 && groups * a.splits > 768;
    pack();
}

hipError_t wkv_launch_paged_attend(const WkvPagedCall& a, int dtype, int head_dim, hipStream_t stream)
{
    const int64_t units = (int64_t)a.c.batch * a.c.kv_heads;
    return by_type(dtype, head_dim, [&](auto t, auto d) {
        using TT = decltype(t);
        constexpr int D = decltype(d)::value;
        const WkvPages& c = a.c;
        const unsigned grid = (unsigned)wkv_paged_groups(a);
        hipError_t e;
        // (a workgroup's start is early where all of them start at once)
        const bool early = c.window == 0 && !a.order;
        if (a.many) e = wkv_launch_paged_flash(a, dtype, head_dim, stream);
        else if (a.starts) e = wkv_launch(&wkv_paged_rows_kernel<TT, D, false, false, false>, grid, THREADS, stream, a);
        else if (early && !a.logits) e = wkv_launch(&wkv_paged_rows_kernel<TT, D, true, true, false>, grid, THREADS, stream, a);
        else if (early) e = wkv_launch(&wkv_paged_rows_kernel<TT, D, true, true, true>, grid, THREADS, stream, a);
        else if (!a.logits) e = wkv_launch(&wkv_paged_rows_kernel<TT, D, true, false, false>, grid, THREADS, stream, a);
        else e = wkv_launch(&wkv_paged_rows_kernel<TT, D, true, false, true>, grid, THREADS, stream, a);
        if (e == hipSuccess && (a.splits > 1 || a.logits)) {
            const int per_tile = (int)std::min<int64_t>(ROWS, (int64_t)a.max_new * a.c.group);
            const int rows = a.splits > 1 ? (int)(units * a.tiles * per_tile) : 0;
            const int per_unit = a.logits ? (int)((wkv_paged_most_keys(a.c, 1) + TALLY - 1) / TALLY) : 0;
            // (More than a few parts: a workgroup a row, or, where there are rows enough to fill the chip, the lanes of a row each all parts:
            // chunks onto 2000 slots of 32 heads on 8: 20 tokens 20.3 | 20.7 us, 40 23.1 | 22.2, 200 39.6 | 30.0.)
            const bool few = a.splits <= FEW, some = !few && a.splits <= SOME && rows >= MANY;
            const int sets = few || some ? THREADS * 4 / D : 1, joins = (rows + sets - 1) / sets;
            const unsigned all = (unsigned)(joins + units * per_unit);
            if (few && a.starts) e = wkv_launch(&wkv_paged_join_few_kernel<TT, D, FEW, false>, all, THREADS, stream, a, joins, rows, per_tile, 1);
            else if (few) e = wkv_launch(&wkv_paged_join_few_kernel<TT, D, FEW, true>, all, THREADS, stream, a, joins, rows, per_tile, per_unit);
            else if (some && a.starts) e = wkv_launch(&wkv_paged_join_few_kernel<TT, D, SOME, false>, all, THREADS, stream, a, joins, rows, per_tile, 1);
            else if (some) e = wkv_launch(&wkv_paged_join_few_kernel<TT, D, SOME, true>, all, THREADS, stream, a, joins, rows, per_tile, per_unit);
            else if (a.starts) e = wkv_launch(&wkv_paged_join_kernel<TT, D, false>, all, THREADS, stream, a, joins, per_tile, 1);
            else e = wkv_launch(&wkv_paged_join_kernel<TT, D, true>, all, THREADS, stream, a, joins, per_tile, per_unit);
        }
        return e;
    });
}

hipError_t wkv_launch_paged_sums(const WkvPagedCall& a, int dtype, int head_dim, hipStream_t stream)
{
    const int64_t units = (int64_t)a.c.batch * a.c.kv_heads;
    const int per_unit = (a.c.max_slots + SUM_KEYS * WAVES - 1) / (SUM_KEYS * WAVES);
    if (dtype != WKV_FP32) return wkv_launch_paged_colsum(a, dtype, head_dim, stream);
    auto go = [&](auto d) {
        constexpr int D = decltype(d)::value;
        for (int64_t u = 0; u < units;) {               // in pieces below 2^32 threads
            const int64_t n = std::min<int64_t>(units - u, ((1 << 24) - 1) / per_unit);
            const hipError_t e = wkv_launch(&wkv_paged_sums_kernel<TF32, D>, (unsigned)(n * per_unit), THREADS, stream, a, (int)u, per_unit);
            if (e != hipSuccess) return e;
            u += n;
        }
        return hipSuccess;
    };
    return head_dim == 64 ? go(std::integral_constant<int, 64>{}) : go(std::integral_constant<int, 128>{});
}
