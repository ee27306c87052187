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
//   wkv_paged_join   the parts of a tile joined; for a step whose weights are summed, the weights of every slot.
//   wkv_paged_sums   the weights of a prefill's rows summed for every slot, from the rows' log-sum-exps.
//   wkv_paged_append new K and V rows into their pages (a step's rows go there inside wkv_paged_rows).
//
// Softmax statistics, sums of the weights and of weight . v are fp32.
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

// The product over 16 dwords of a row (a lane's KL loads): 16-bit rows 8 elements a load and instruction, fp32 rows 4 a load.
template <class TT, int KL> __device__ __forceinline__ f32x4_t dot_tile(const u32x4_t (&a)[KL], const u32x4_t (&b)[KL])
{
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KL; ++kk) {
        if constexpr (TT::BYTES == 2) {
            s = mfma<TT>(a[kk], b[kk], s);
        } else {
            const f32x4_t x = __builtin_bit_cast(f32x4_t, a[kk]), y = __builtin_bit_cast(f32x4_t, b[kk]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = mfma_f32(x[e], y[e], s);
        }
    }
    return s;
}

template <class TT, int D> struct Frag {
    using S = Shape<TT, D>;
    u32x4_t k[S::NT][S::KL];
    uint32_t v[S::VK][S::NH][S::VW];
};

template <class TT, int D>
__global__ __launch_bounds__(THREADS, (D * TT::BYTES > 256) ? 1 : 2)
void wkv_paged_rows_kernel(const WkvPagedCall a)
{
    using S = Shape<TT, D>;
    constexpr int BK = S::BK, NT = S::NT, KL = S::KL, VK = S::VK, VE = S::VE, NH = S::NH, VW = S::VW;
    __shared__ float s_m[WAVES][ROWS], s_l[WAVES][ROWS];
    __shared__ float s_o[WAVES][ROWS][16 * VE + 4];

    int id = blockIdx.x;
    const int part = id % a.splits; id /= a.splits;
    const int tile = id % a.tiles;
    const int unit = id / a.tiles;
    Tile t;
    if (!unit_of(a, unit, tile * ROWS, t)) return;
    const int group = a.c.group;
    const int r0 = tile * ROWS, r1 = min(t.rows, r0 + ROWS);
    const int p_lo = t.pos0 + r0 / group, p_hi = t.pos0 + (r1 - 1) / group;
    const Span sp = span(a, p_lo, p_hi);
    if (part >= sp.parts) return;
    const int begin = part * sp.per, end = min(sp.blocks, begin + sp.per);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const WkvPages& c = a.c;
    const int window = c.window > 0 ? c.window : 0x40000000;

    // a step appends its row; nothing reads it from the page in this launch
    const bool append = a.starts == nullptr && a.k_new != nullptr;
    const int pos_new = append ? p_lo : -1;
    const char* new_k = a.k_new + t.b * a.k_bytes + t.h * a.k_head;
    const char* new_v = a.v_new + t.b * a.v_bytes + t.h * a.v_head;
    if (append && part == 0 && tile == 0 && wave == WAVES - 1 && pos_new >= 0) {
        const int page = c.table[t.b * c.table_stride + (pos_new >> c.page_shift)];
        if ((unsigned)page < (unsigned)c.n_pages && lane < D * TT::BYTES / 16) {
            const int64_t at = page * c.page_bytes + (pos_new & ((1 << c.page_shift) - 1)) * c.slot_bytes + t.h * c.head_bytes + lane * 16;
            *reinterpret_cast<u32x4_t*>(c.k + at) = reinterpret_cast<const u32x4_t*>(new_k)[lane];
            *reinterpret_cast<u32x4_t*>(c.v + at) = reinterpret_cast<const u32x4_t*>(new_v)[lane];
        }
    }

    // the lane's row: its position, its query as the second operand of K Q^T
    const int row = r0 + col;
    const bool row_ok = row < r1;
    const int token = min(row, r1 - 1) / group;
    const int p_row = row_ok ? t.pos0 + token : -1;
    u32x4_t q[KL];
    {
        const int head = t.h * group + min(row, r1 - 1) - token * group;
        const char* src = a.q + (t.q.row0 + token) * a.q_bytes + head * a.q_head + g * 16;
#pragma unroll
        for (int kk = 0; kk < KL; ++kk) q[kk] = *reinterpret_cast<const u32x4_t*>(src + kk * 64);
    }
    const char* kbase = c.k + t.h * c.head_bytes + g * 16;
    const char* vbase = c.v + t.h * c.head_bytes + col * (VE * TT::BYTES);
    const int in_page = (1 << c.page_shift) - 1;

    auto slot_of = [&](int blk) { const int i = blk * BK; return i < sp.first ? i : i - sp.first + sp.lo; };
    // page of the tile of 16 slots from `pos` on, as the table says, and -1 for what is none
    const int32_t* table = c.table + t.b * c.table_stride;
    auto entry = [&](int pos) { return load_uniform(table + min(pos >> c.page_shift, c.max_pages - 1)); };
    auto page_of = [&](int pos, int page) { return (unsigned)page < (unsigned)c.n_pages && pos < c.max_slots ? page : -1; };

    float m, l;
    f32x4_t o[NH][VE];
    bool careful = false;

    Frag<TT, D> f[2];
    // Pages that are not there are loaded as page 0 (it is in the pool) and masked.
    auto load = [&](Frag<TT, D>& x, int pos, const int (&pages)[NT]) {
        const char* kr[NT];
        const char* vr[VK];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int64_t at = max(pages[i], 0) * c.page_bytes;
            const int pk = pos + i * 16 + col;
            kr[i] = kbase + at + (pk & in_page) * c.slot_bytes;
            if (pk == pos_new) kr[i] = new_k + g * 16;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int pv = pos + i * 16 + g * 4 + j;
                vr[i * 4 + j] = vbase + at + (pv & in_page) * c.slot_bytes;
                if (pv == pos_new) vr[i * 4 + j] = new_v + col * (VE * TT::BYTES);
            }
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int kk = 0; kk < KL; ++kk) x.k[i][kk] = *reinterpret_cast<const u32x4_t*>(kr[i] + kk * 64);
#pragma unroll
        for (int j = 0; j < VK; ++j)
#pragma unroll
            for (int h = 0; h < NH; ++h) load_words<VW>(vr[j] + h * (16 * VE * TT::BYTES), x.v[j][h]);
    };

    auto use = [&](Frag<TT, D>& x, int pos, const int (&pages)[NT]) {
        f32x4_t s[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) s[i] = dot_tile<TT, KL>(x.k[i], q);
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
                    // values that no row sees have no effect, whatever they are
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
        if (a.logits && row_ok) {
            float* dst = a.logits + ((int64_t)unit * group + row) * a.logit_stride + pos + g * 4;
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
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int e = 0; e < VE; ++e) o[h][e] *= f0;
        }
        const float ref = (m == -INFINITY ? 0.f : m) + BIAS<TT>;
        float p[NT][4];
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[i][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][j], a.scale, -ref));
                l += p[i][j];
            }
        if (careful) {
            // one key after the other, each row what it sees, weights in fp32
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll 1
                    for (int gs = 0; gs < 4; ++gs) {
                        const float w = __shfl(p[i][j], gs * 16 + col);
                        const int pk = pos + i * 16 + gs * 4 + j;
                        if (pages[i] >= 0 && pk <= p_row && (pk > p_row - window || pk < c.n_sink)) {
                            const char* src = c.v + t.h * c.head_bytes + pages[i] * c.page_bytes + (pk & in_page) * c.slot_bytes;
#pragma unroll
                            for (int h = 0; h < NH; ++h)
#pragma unroll
                                for (int r = 0; r < 4; ++r)
#pragma unroll
                                    for (int e = 0; e < VE; ++e)
                                        o[h][e][r] += w * load_elem<TT>(src, h * 16 * VE + (g * 4 + r) * VE + e);
                        }
                    }
            return;
        }
        if constexpr (S::HALF) {
            // The weights as a sum of two 16-bit numbers: what is left of them is below 2^-16 (bf16) of a weight.  One number
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
                    u32x4_t vt = {};          // element e of the lane's keys
#pragma unroll
                    for (int w = 0; w < VK / 2; ++w)
                        vt[w] = __builtin_amdgcn_perm(x.v[2 * w + 1][h][e / 2], x.v[2 * w][h][e / 2], (e & 1) ? 0x07060302u : 0x05040100u);
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
    };

    // The wave's blocks: begin + wave, and every fourth from there.  The next block travels while one is used; behind the
    // last one the last is loaded again (a load that is there on every path is what the waits are counted by).
    const int count = begin + wave < end ? (end - begin - wave + WAVES - 1) / WAVES : 0;
    int pos[3] = {0, 0, 0}, pages[3][NT];          // of the block in use, the one that travels, the one after it
    auto ahead = [&](int k, int& p, int (&e)[NT]) {
        p = __builtin_amdgcn_readfirstlane(slot_of(begin + wave + WAVES * min(k, count - 1)));
#pragma unroll
        for (int i = 0; i < NT; ++i) e[i] = entry(p + i * 16);
    };
    auto known = [&](int p, int (&e)[NT]) {
#pragma unroll
        for (int i = 0; i < NT; ++i) e[i] = page_of(p + i * 16, e[i]);
    };
    auto shift = [&] {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            pos[x] = pos[x + 1];
#pragma unroll
            for (int i = 0; i < NT; ++i) pages[x][i] = pages[x + 1][i];
        }
    };
    for (;;) {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int e = 0; e < VE; ++e) o[h][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (count > 0) {
            ahead(0, pos[0], pages[0]);
            ahead(1, pos[1], pages[1]);
            known(pos[0], pages[0]);
            load(f[0], pos[0], pages[0]);
            for (int k = 0; k < count; k += 2) {
                known(pos[1], pages[1]);
                load(f[1], pos[1], pages[1]);
                ahead(k + 2, pos[2], pages[2]);
                use(f[0], pos[0], pages[0]);
                if (k + 1 >= count) break;
                shift();
                known(pos[1], pages[1]);
                load(f[0], pos[1], pages[1]);
                ahead(k + 3, pos[2], pages[2]);
                use(f[1], pos[0], pages[0]);
                shift();
            }
        }
        // A value that is not finite spoils the matrix product: it meets weights of 0 of rows that do not see it, and parts of weights
        // that are 0 or negative.  Sums stay finite otherwise, so if one has not the wave goes over its blocks again, key by key.
        float z = 0.f;
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int e = 0; e < VE; ++e)
#pragma unroll
                for (int r = 0; r < 4; ++r) z = __builtin_fmaf(o[h][e][r], 0.f, z);
        if (careful || !__any(z != 0.f)) break;           // (0 x infinity and 0 x NaN are NaN, which is no 0)
        careful = true;
    }

    // ---- the four waves' sums joined
    l = rows_sum(l);
    if (g == 0) { s_m[wave][col] = m; s_l[wave][col] = l; }
    __syncthreads();
    float top = s_m[0][col];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, s_m[w][col]);
    const float mine = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    const bool direct = sp.parts == 1;
    const int orow = threadIdx.x >> 4, piece = threadIdx.x & 15;           // 16 lanes write a row
    float sum = 0.f, otop = s_m[0][orow];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) otop = fmaxf(otop, s_m[w][orow]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += s_m[w][orow] == -INFINITY ? s_l[w][orow] : s_l[w][orow] * __builtin_amdgcn_exp2f(s_m[w][orow] - otop);
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    const int64_t cell = ((int64_t)unit * a.tiles + tile) * a.splits + part;
    const int otoken = min(r0 + orow, r1 - 1) / group, ohead = t.h * group + min(r0 + orow, r1 - 1) - otoken * group;
    char* dst = a.out + (t.q.row0 + otoken) * a.out_bytes + ohead * a.out_head;
#pragma unroll
    for (int h = 0; h < NH; ++h) {
        if (h > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < VE; ++e) s_o[wave][col][(g * 4 + r) * VE + e] = o[h][e][r] * mine;
        __syncthreads();
        float x[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            x[e] = s_o[0][orow][piece * VE + e];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) x[e] += s_o[w][orow][piece * VE + e];
        }
        if (direct) {
            if (r0 + orow < r1) {
                uint32_t w[VW];
#pragma unroll
                for (int e = 0; e < VW; ++e) {
                    if constexpr (S::HALF) w[e] = pack2<TT>(mean<TT>(x[2 * e], inv), mean<TT>(x[2 * e + 1], inv));
                    else w[e] = __builtin_bit_cast(uint32_t, mean<TT>(x[e], inv));
                }
                store_words<VW>(dst + (h * 16 + piece) * (VE * TT::BYTES), w);
            }
        } else {
            float* p = a.part + (cell * ROWS + orow) * D + (h * 16 + piece) * VE;
#pragma unroll
            for (int e = 0; e < VE; e += 4) *reinterpret_cast<f32x4_t*>(p + e) = f32x4_t{x[e], x[e + 1], x[e + 2], x[e + 3]};
        }
    }
    if (piece == 0) {
        if (a.ml) { a.ml[cell * 32 + orow] = otop; a.ml[cell * 32 + 16 + orow] = sum; }
        if (a.lse && direct && r0 + orow < r1)
            a.lse[(int64_t)(t.q.row0 + otoken) * (c.kv_heads * group) + ohead] = otop == -INFINITY ? INFINITY : otop + BIAS<TT> + __builtin_amdgcn_logf(sum);
    }
}

// ---------------------------------------------------------------- joining
constexpr int TALLY = 1024;          // slots whose weights one workgroup sums

// Workgroup x: tile x / per_tile.  The first of a tile joins its parts; with logits, every one sums the weights of TALLY of the
// keys that the step saw, in the order of span().
template <class TT, int D>
__global__ __launch_bounds__(THREADS)
void wkv_paged_join_kernel(const WkvPagedCall a, int per_tile)
{
    using S = Shape<TT, D>;
    const int cell = blockIdx.x / per_tile, piece = blockIdx.x - cell * per_tile;
    const int unit = cell / a.tiles, tile = cell - unit * a.tiles;
    Tile t;
    if (!unit_of(a, unit, tile * ROWS, t)) return;
    const int group = a.c.group, r0 = tile * ROWS, r1 = min(t.rows, r0 + ROWS);
    // the keys were cut into parts for a tile of a.tile_rows rows
    const int t0 = r0 & -a.tile_rows, t1 = min(t.rows, t0 + a.tile_rows);
    const int p_lo = t.pos0 + t0 / group, p_hi = t.pos0 + (t1 - 1) / group;
    const Span sp = span(a, p_lo, p_hi);

    const int row = threadIdx.x >> 4, lane = threadIdx.x & 15;
    if (piece == 0 && sp.parts > 1 && r0 + row < r1) {
        const float* ml = a.ml + (int64_t)cell * a.splits * 32 + row;
        float top = -INFINITY, sum = 0.f;
        for (int s = 0; s < sp.parts; ++s) top = fmaxf(top, ml[s * 32]);
        constexpr int N = D / 64;                                          // four elements each
        f32x4_t x[N] = {};
        const float* part = a.part + ((int64_t)cell * a.splits * ROWS + row) * D + lane * 4;
        for (int s = 0; s < sp.parts; ++s) {
            const float f = ml[s * 32] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[s * 32] - top);
            sum += f * ml[s * 32 + 16];
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] += f * *reinterpret_cast<const f32x4_t*>(part + (int64_t)s * ROWS * D + i * 64);
        }
        const float inv = sum != 0.f ? 1.f / sum : 0.f;
        const int token = (r0 + row) / group, head = t.h * group + r0 + row - token * group;
        char* dst = a.out + (t.q.row0 + token) * a.out_bytes + head * a.out_head;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (S::HALF)
                *reinterpret_cast<uint2*>(dst + (i * 16 + lane) * 8) = make_uint2(pack2<TT>(mean<TT>(x[i][0], inv), mean<TT>(x[i][1], inv)),
                                                                              pack2<TT>(mean<TT>(x[i][2], inv), mean<TT>(x[i][3], inv)));
            else
                *reinterpret_cast<f32x4_t*>(dst + (i * 16 + lane) * 16) = f32x4_t{mean<TT>(x[i][0], inv), mean<TT>(x[i][1], inv), mean<TT>(x[i][2], inv), mean<TT>(x[i][3], inv)};
        }
        if (a.lse && lane == 0)
            a.lse[(int64_t)(t.q.row0 + token) * (a.c.kv_heads * group) + head] = top == -INFINITY ? INFINITY : top + BIAS<TT> + __builtin_amdgcn_logf(sum);
    }
    if (!a.logits) return;

    // a step: every row of the unit is of one token; tile 0's workgroups sum over all of them
    if (tile != 0) return;
    const int keys = p_hi < 0 ? 0 : sp.first + p_hi + 1 - sp.lo;
    const int first = piece * TALLY;
    if (first >= keys) return;
    float w[TALLY / THREADS] = {};
    for (int r = 0; r < group; ++r) {
        const float* ml = a.ml + ((int64_t)unit * a.tiles + r / ROWS) * a.splits * 32 + r % ROWS;
        float top = -INFINITY, sum = 0.f;
        for (int s = 0; s < sp.parts; ++s) top = fmaxf(top, ml[s * 32]);
        for (int s = 0; s < sp.parts; ++s)
            sum += ml[s * 32 + 16] * (ml[s * 32] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[s * 32] - top));
        const float lse = top == -INFINITY ? INFINITY : top + BIAS<TT> + __builtin_amdgcn_logf(sum);
        const float* lg = a.logits + ((int64_t)unit * group + r) * a.logit_stride;
#pragma unroll
        for (int i = 0; i < TALLY / THREADS; ++i) {
            const int j = first + i * THREADS + threadIdx.x;
            if (j < keys) w[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(lg[j < sp.first ? j : j - sp.first + sp.lo], a.scale, -lse));
        }
    }
    float* sc = a.c.scores + (int64_t)unit * a.c.score_stride;
#pragma unroll
    for (int i = 0; i < TALLY / THREADS; ++i) {
        const int j = first + i * THREADS + threadIdx.x;
        if (j >= keys) continue;
        const int p = j < sp.first ? j : j - sp.first + sp.lo;
        if (p == p_hi && a.k_new) sc[p] = w[i];
        else sc[p] += w[i];
    }
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
    if (!unit_of(a, unit, 0, t)) return;
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

// ---------------------------------------------------------------- appending a chunk
__global__ __launch_bounds__(THREADS)
void wkv_paged_append_kernel(const WkvPagedCall a, int row_chunks, int per_seq)
{
    const WkvPages& c = a.c;
    const int b = blockIdx.x / per_seq;
    const Seq s = sequence(a, b);
    const int64_t i = (int64_t)(blockIdx.x - b * per_seq) * THREADS + threadIdx.x;
    const int per_token = row_chunks * c.kv_heads;
    const int token = (int)(i / per_token), rest = (int)(i - (int64_t)token * per_token);
    const int pos = s.len - s.n + token;
    if (token >= s.n || pos < 0) return;
    const int page = c.table[b * c.table_stride + (pos >> c.page_shift)];
    if ((unsigned)page >= (unsigned)c.n_pages) return;
    const int h = rest / row_chunks, x = rest - h * row_chunks;
    const int64_t to = page * c.page_bytes + (pos & ((1 << c.page_shift) - 1)) * c.slot_bytes + h * c.head_bytes + x * 16;
    const u32x4_t k = *reinterpret_cast<const u32x4_t*>(a.k_new + (s.row0 + token) * a.k_bytes + h * a.k_head + x * 16);
    const u32x4_t v = *reinterpret_cast<const u32x4_t*>(a.v_new + (s.row0 + token) * a.v_bytes + h * a.v_head + x * 16);
    *reinterpret_cast<u32x4_t*>(c.k + to) = k;
    *reinterpret_cast<u32x4_t*>(c.v + to) = v;
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

void wkv_paged_shape(WkvPagedCall& a, int64_t units, int64_t rows, int64_t most, int dtype, int head_dim)
{
    a.tiles = (int)((rows + ROWS - 1) / ROWS);
    a.many = dtype != WKV_FP32 && rows > 32;
    a.tile_rows = a.many ? 128 : ROWS;
    a.block = a.many ? (head_dim > 128 ? 32 : 64) : dtype == WKV_FP32 || head_dim > 128 ? 16 : 32;
    a.least = WAVES;
    const int64_t groups = units * ((rows + a.tile_rows - 1) / a.tile_rows), part = (int64_t)a.block * a.least;
    a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(512 + groups - 1) / groups, (most + part - 1) / part, 64}));
}

hipError_t wkv_launch_paged_append(const WkvPagedCall& a, int dtype, int head_dim, hipStream_t stream)
{
    const int row_chunks = head_dim * (dtype == WKV_FP32 ? 4 : 2) / 16;
    const int64_t per_seq = ((int64_t)a.max_new * a.c.kv_heads * row_chunks + THREADS - 1) / THREADS;
    // in pieces of whole sequences, each launch below 2^32 threads: nothing but the sequence's number depends on the piece
    for (int b0 = 0; b0 < a.c.batch;) {
        const int n = (int)std::min<int64_t>(a.c.batch - b0, std::max<int64_t>(1, ((1 << 24) - 1) / per_seq));
        if (per_seq >= 1 << 24) return hipErrorInvalidValue;
        WkvPagedCall p = a;
        p.c.batch = n;
        p.c.lens += b0;
        p.c.table += b0 * p.c.table_stride;
        p.starts += b0;
        hipLaunchKernelGGL(wkv_paged_append_kernel, dim3((unsigned)(n * per_seq)), dim3(THREADS), 0, stream, p, row_chunks, (int)per_seq);
        b0 += n;
    }
    return hipGetLastError();
}

hipError_t wkv_launch_paged_attend(const WkvPagedCall& a, int dtype, int head_dim, hipStream_t stream)
{
    const int64_t units = (int64_t)a.c.batch * a.c.kv_heads;
    return by_type(dtype, head_dim, [&](auto t, auto d) {
        using TT = decltype(t);
        constexpr int D = decltype(d)::value;
        hipError_t e;
        if (a.many) {
            e = wkv_launch_paged_flash(a, dtype, head_dim, stream);
        } else {
            hipLaunchKernelGGL((wkv_paged_rows_kernel<TT, D>), dim3((unsigned)(units * a.tiles * a.splits)), dim3(THREADS), 0, stream, a);
            e = hipGetLastError();
        }
        if (e == hipSuccess && (a.splits > 1 || a.logits)) {
            const int per_tile = a.logits ? (int)((a.c.max_slots + 64 + TALLY - 1) / TALLY) : 1;
            hipLaunchKernelGGL((wkv_paged_join_kernel<TT, D>), dim3((unsigned)(units * a.tiles * per_tile)), dim3(THREADS), 0, stream, a, per_tile);
            e = hipGetLastError();
        }
        return e;
    });
}

hipError_t wkv_launch_paged_sums(const WkvPagedCall& a, int dtype, int head_dim, hipStream_t stream)
{
    const int64_t units = (int64_t)a.c.batch * a.c.kv_heads;
    const int per_unit = (a.c.max_slots + SUM_KEYS * WAVES - 1) / (SUM_KEYS * WAVES);
    return by_type(dtype, head_dim, [&](auto t, auto d) {
        using TT = decltype(t);
        constexpr int D = decltype(d)::value;
        for (int64_t u = 0; u < units;) {               // in pieces below 2^32 threads
            const int64_t n = std::min<int64_t>(units - u, ((1 << 24) - 1) / per_unit);
            hipLaunchKernelGGL((wkv_paged_sums_kernel<TT, D>), dim3((unsigned)(n * per_unit)), dim3(THREADS), 0, stream, a, (int)u, per_unit);
            u += n;
        }
        return hipGetLastError();
    });
}
