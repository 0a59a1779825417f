// Attention over the paged 8-bit cache for sequences that share a prefix, which is read once for all of them.
//
// softmax(q k^T) v over keys that lie in parts joins from the parts' maxima, weights and sums: m = max m_i, l = sum l_i 2^(m_i - m),
// o = sum o_i 2^(m_i - m), out = o / l.  The shared part of a group (its positions below S = shared / 64 * 64, whole steps) is visited with
// the rows of all its sequences in tiles of 128: a step's codes are read and decoded once for 128 rows, as for a piece of a prompt
// (many_steps).  What a sequence has behind it is visited with its own rows in tiles of 16 or 32, a wave by itself to each tile, or to a part of its
// steps: such parts are short, and waves that wait for each other would wait more than they work.  One launch does both: the
// first is bound by matrix and vector work, the second by the bytes of the cache, and workgroups of both kinds share the CUs.  A second one
// joins.  How long the sequences are is on the device alone: each workgroup finds its part of the work by itself (3 us of a call, 4 to 5 with 256
// sequences, and from there on by the number of workgroups times that of sequences and groups: some 250 of 515 us with 4096 sequences of one group).
//
// A CU holds two workgroups.  A step of a prefix takes one 1.6 us by itself and 2.3 beside another (1.15 per step), as its matrix and vector
// work take turns then; beside sequences' own parts, which wait for memory, 1.7.
//
// Measured, 32 query and 8 kv heads, D = 128, E4M3, one token per sequence, call to call: 64 sequences of up to 512 behind 8192 33.5 us (dma_cache_attn,
// which reads the prefix 64 times, by way of the caches, 105); 256 of up to 700 behind 32768 203 us = 0.68 PFLOP/s (1845; the matrix product of
// 8192^3 would take 121 for as many flops); 64 of up to 500 behind 8192 with 32 kv heads 65 us for 217 MB = 3.3 TB/s (538); 32 under a window of 4096
// 35.5 us (39.6).  Of the 33.5: 3 to find the work, 3.5 until the first products, 8 steps of the prefix 14.5 (own parts end before), 2 to write pieces, 2.8
// launch and end, the join 6.5.
#include "dma_cache_many.hpp"
#include <algorithm>

namespace dma {

constexpr int GROUPS_LDS = 512;              // groups whose bounds are kept in LDS
constexpr int ROWS_MANY = 128;
constexpr int WAVES = 4;

struct SharedArgs {
    CacheAttnArgs a;         // pieces and split (first piece, how many): of what the sequences have to themselves, per tile of 16 * MT rows
    Groups g;
    int rows_per_seq;        // query rows of a kv head and sequence: N * G
    int piece_rows;          // of a sequence's own piece: at most 16 * MT
    int piece_size;          // in floats: sums, then maxima and weights, up to a multiple of 4
    float* pieces;           // of the prefixes: per workgroup [128][D] sums, [128] maxima, [128] weights
    int4* where;             // per sequence and kv head, for the tile that holds its first rows and the next one: first piece, how many (0: it
                             // shares nothing), place of the sequence's first row in the tile
    int64_t max_pieces, max_own;
    int cus;
    int more_own;            // waves beyond one for each row tile of the sequences: tiles in several parts
};

struct Bounds {
    int lo, hi;              // sequences
    int steps;               // that they share
};
DMA_DEV int shared_steps(const SharedArgs& x, int shared) { return max(min(shared, x.a.capacity), 0) / STEP; }

// The group of sequence b: the last one that does not begin behind it.  first(g): where group g begins.
template <typename F>
DMA_DEV int group_of(const F& first, int n, int b)
{
    int lo = 0, hi = n;                      // the answer + 1 is in [lo, hi]
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (first(mid) <= b) lo = mid + 1;
        else hi = mid;
    }
    return lo > 0 && b < first(lo) ? lo - 1 : -1;
}

// A sequence, and the first step that it does not share.
struct OwnSeq {
    int start, n, own;
};

// The steps that a row tile of a sequence visits behind what it shares: [own, own + sink_steps) and [first, first + steps - sink_steps).
struct OwnRange {
    int own, sink_steps, first, steps;
    DMA_DEV int position(int j) const { return (j < sink_steps ? own + j : first + j - sink_steps) * STEP; }
};
// (A start behind the table is brought to its end: what that lets in too much is not seen by any row.)
template <int ROWS, bool ONE>
DMA_DEV OwnRange own_range(const CacheAttnArgs& a, const OwnSeq& q, int tile)
{
    const int start = min(q.start, a.capacity), from = start + (ONE ? 0 : token_of<true>(a, tile * ROWS));
    const int hi = min(start + 1 + (ONE ? q.n - 1 : min(q.n - 1, token_of<true>(a, tile * ROWS + ROWS - 1))), a.capacity);
    const int lo = a.window ? min(max(from - a.window + 1, 0), hi) : 0;
    OwnRange r;
    r.own = q.own;
    r.first = max(lo / STEP, q.own);
    r.sink_steps = max((min(a.sinks, hi) + STEP - 1) / STEP - q.own, 0);
    if (q.own + r.sink_steps >= r.first) {
        r.sink_steps = 0;
        r.first = q.own;
    }
    r.steps = max(r.sink_steps + (hi + STEP - 1) / STEP - r.first, 0);
    return r;
}

DMA_DEV int wave_scan(int x)                 // the sum up to and with this lane's
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);       // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);       // row_bcast:15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
DMA_DEV int wave_max(int x)
{
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x111, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x112, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x114, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x118, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x142, 0xa, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(x, 63);
}
// The sum over the lanes.  In binary32: how work is divided needs no more, and every wave adds in the same order.
DMA_DEV float wave_sum(float v)
{
#define DMA_SHIFTED(ctrl, rows) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, false))
    v += DMA_SHIFTED(0x111, 0xf);
    v += DMA_SHIFTED(0x112, 0xf);
    v += DMA_SHIFTED(0x114, 0xf);
    v += DMA_SHIFTED(0x118, 0xf);
    v += DMA_SHIFTED(0x142, 0xa);
    v += DMA_SHIFTED(0x143, 0xc);
#undef DMA_SHIFTED
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// One workgroup's part of the prefixes: 128 rows of a group, some of their steps, into piece `piece`: of those of part `part` of `parts` the first
// share `early`, or (late) the others.  pieces: the first one of the rows, and how many.
template <int D, bool E5M2, bool UNI>
DMA_DEV void prefix_part(const SharedArgs& x, const ManyLds<D>& lds, int (&ends)[5][WAVES], const Bounds& g, int h, int tile, int part, int parts, float early, bool late, int64_t piece, int2 pieces)
{
    const CacheAttnArgs& a = x.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int64_t all_rows = (int64_t)(g.hi - g.lo) * x.rows_per_seq;
    const int rows = (int)min(all_rows - (int64_t)tile * ROWS_MANY, (int64_t)ROWS_MANY), my_rows = min(rows - wave * 32, 32);
    // ---- this lane's row: sequence, token and head
    const int64_t r = min((int64_t)tile * ROWS_MANY + wave * 32 + col, all_rows - 1);
    const int b = g.lo + (int)((unsigned)r / (unsigned)x.rows_per_seq), in_seq = (int)((unsigned)r % (unsigned)x.rows_per_seq);
    const int tok = token_of<true>(a, in_seq), place = wave * 32 + col;
    if (part == 0 && !late && half == 0 && col < my_rows && (in_seq == 0 || place == 0))
        x.where[((int64_t)b * a.c.Hkv + h) * 2 + (in_seq != 0)] = make_int4(pieces.x, pieces.y, place - in_seq, 0);
    v8bf qf[D / 16];
    {
        const char* qp = a.q.data + b * a.q.stride_batch + (h * a.G + in_seq - tok * a.G) * a.q.stride_head + tok * a.q.stride_token;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const v8bf*)(qp + (ks * 16 + half * 8) * 2);
    }
    const SeqInfo sq = seq_of(a, b);
    const bool exists = tok < sq.n && col < my_rows;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)                           // (rows that do not exist may hold anything, and share the wave's maxima)
        qf[ks] = exists ? qf[ks] : __builtin_bit_cast(v8bf, v4i{0, 0, 0, 0});
    // ---- what is visible.  Rows that do not exist have no say in it
    const int64_t at = (int64_t)sq.start + tok;
    ManyRows view;
    view.my_rows = my_rows;
    view.vis_hi = exists ? cut_position(at) : -1;
    view.vis_lo = exists && a.window ? cut_position(at - a.window + 1) : 0;
    view.all_hi = -wave_max(exists ? -view.vis_hi : -POS_MAX);
    view.some_hi = wave_max(view.vis_hi);
    view.all_lo = wave_max(view.vis_lo);
    view.some_lo = -wave_max(exists ? -view.vis_lo : -POS_MAX);
    // the table of the first sequence that has tokens: one that ended may have none of the pages any more
    const int first_b = wave_max(exists ? -b : -0x7fffffff);
    if (lane == 0) {
        ends[4][wave] = first_b;
        ends[0][wave] = view.all_hi;
        ends[1][wave] = view.some_hi;
        ends[2][wave] = view.all_lo;
        ends[3][wave] = view.some_lo;
    }
    __syncthreads();
    view.wg_hi = min(min(ends[0][0], ends[0][1]), min(ends[0][2], ends[0][3]));
    view.any_hi = max(max(ends[1][0], ends[1][1]), max(ends[1][2], ends[1][3]));
    view.wg_lo = max(max(ends[2][0], ends[2][1]), max(ends[2][2], ends[2][3]));
    view.any_lo = min(min(ends[3][0], ends[3][1]), min(ends[3][2], ends[3][3]));
    view.wg_hi = __builtin_amdgcn_readfirstlane(view.wg_hi);
    view.any_hi = __builtin_amdgcn_readfirstlane(view.any_hi);
    view.wg_lo = __builtin_amdgcn_readfirstlane(view.wg_lo);
    view.any_lo = __builtin_amdgcn_readfirstlane(view.any_lo);
    const int by = min(-__builtin_amdgcn_readfirstlane(max(max(ends[4][0], ends[4][1]), max(ends[4][2], ends[4][3]))), a.s.B - 1);
    // ---- the steps: of the shared ones, those that a row sees
    const int hi = min(view.any_hi + 1, g.steps * STEP), lo = min(view.any_lo, hi);
    StepRange range;
    range.first = lo / STEP;
    range.sink_steps = (min(a.sinks, hi) + STEP - 1) / STEP;
    if (range.sink_steps >= range.first) range.sink_steps = range.first = 0;
    range.steps = range.sink_steps + (hi + STEP - 1) / STEP - range.first;
    int begin = (int)((int64_t)range.steps * part / parts), end = (int)((int64_t)range.steps * (part + 1) / parts);
    const int cut = min(begin + __builtin_amdgcn_readfirstlane((int)ceilf((float)(end - begin) * early)), end);
    (late ? begin : end) = cut;
    v16f o[D / 32];
    float m, l;
    many_steps<D, E5M2, WAVES, UNI, true>(a, lds, by, h, range, begin, end, view, qf, o, m, l);
    if (col >= my_rows) return;
    l = cross_half_sum(l);
    float* p = x.pieces + piece * (ROWS_MANY * (D + 2));          // (past the caches, which would be written back at the kernel's end: 29.5 us, 27.9)
    const int rr = wave * 32 + col;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            __builtin_nontemporal_store(v4f{o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]}, (v4f*)(p + rr * D + dt * 32 + 8 * q + 4 * half));
    if (half == 0) {
        p[ROWS_MANY * D + rr] = m;
        p[ROWS_MANY * D + ROWS_MANY + rr] = l;
    }
}

// One wave's part of what a sequence has to itself: steps [begin, end) for a tile of 16 * MT of its rows, into a piece.  S^T = K Q^T with the keys in
// an order that leaves every probability in the lane that needs it for O^T = V^T P^T, one maximum per row that is raised only where it was far too
// low, codes of the next step on their way while one is worked on: as in the kernel for few rows (dma_cache_attn.hip), whose comments say why.  (Its loop
// written once more: as one function for both, that kernel's instructions changed.  What is mended in one is mended in the other.)
// qs: with 32 rows, room for the queries' operands in LDS.
template <int D, bool E5M2, int MT, bool UNI>
DMA_DEV void own_part(const SharedArgs& x, const OwnSeq& sq, const OwnRange& range, int b, int h, int tile, int begin, int end, int64_t piece, v8bf* qs)
{
    constexpr int ROWS = 16 * MT, KJ = D / 64, DT = D / 16;
    const CacheAttnArgs& a = x.a;
    const CacheView& c = a.c;
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4, page_mask = (1 << c.page_shift) - 1;
    const int rows = min(sq.n * a.G - tile * ROWS, ROWS);
    const int* table = c.page_table + (int64_t)b * c.max_pages;
    // ---- pages and codes of a step: of the 16 positions whose keys this lane loads, and of those whose values it loads
    auto page_of = [&](int j, int g) -> int {
        const int at = min((range.position(j) + (UNI ? 0 : 16 * g)) >> c.page_shift, c.max_pages - 1);
        return UNI ? scalar_at(table, __builtin_amdgcn_readfirstlane(at)) : table[at];
    };
    auto there = [&](int page, int j, int g) -> int {             // looked at where it is used: looking at once would wait for the codes too
        if constexpr (!UNI) asm volatile("" : "+v"(page));
        return (range.position(j) + (UNI ? 0 : 16 * g)) >> c.page_shift < c.max_pages ? page : -1;
    };
    auto slab_of = [&](int page) -> int64_t {
        if constexpr (UNI) page = __builtin_amdgcn_readfirstlane(page);
        return (int64_t)((unsigned)page < c.page_limit ? page : 0) * c.Hkv + h;
    };
    v4i kr[4][KJ], vr[DT];
    uint8_t k_scale = 0, v_scale = 0;
    int v_page = -1;
    // the positions of a lane's keys: 16 (col / 4) + 4 t + col % 4 in product t
    auto load_k = [&](int j, int page, bool on) {
        const int64_t slab = slab_of(page);
        const int pos = range.position(j), at = 16 * (col >> 2);
        const uint8_t* base = c.k_codes + ((slab << c.page_shift) + ((UNI ? pos : pos + at) & page_mask)) * D;
        const uint8_t* p = base + (on ? (unsigned)(((UNI ? at : 0) + (col & 3)) * D + grp * 16) : 0u);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < KJ; ++i) kr[t][i] = *(const v4i*)(p + t * 4 * D + i * 64);
        k_scale = c.k_scales[slab];
    };
    auto load_v = [&](int j, int page, bool on) {
        const int64_t slab = slab_of(page);
        const int pos = range.position(j);
        const uint8_t* base = c.v_codes + ((slab * D) << c.page_shift) + ((UNI ? pos : pos + 16 * grp) & page_mask);
        const unsigned mine = on ? (col << c.page_shift) + (UNI ? 16 * grp : 0) : 0u;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vr[dt] = *(const v4i*)(base + ((dt * 16) << c.page_shift) + mine);
        v_scale = c.v_scales[slab];
        v_page = page;
    };
    int pk = -1, pv = -1;                                         // pages of the step after the next
    if (begin < end) {
        pk = page_of(begin, col >> 2);
        pv = UNI ? pk : page_of(begin, grp);
    }
    // ---- rows
    v8bf qf[MT][2 * KJ];
    int vis_lo[MT], vis_hi[MT];                                   // what the row of this lane's column sees: these positions and those below sinks
    const int64_t from = sq.start;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = min(mt * 16 + col, rows - 1) + tile * ROWS, i = token_of<true>(a, r);
        const char* qp = a.q.data + b * a.q.stride_batch + (h * a.G + r - i * a.G) * a.q.stride_head + i * a.q.stride_token;
#pragma unroll
        for (int ks = 0; ks < 2 * KJ; ++ks) qf[mt][ks] = *(const v8bf*)(qp + ((ks >> 1) * 64 + grp * 16 + (ks & 1) * 8) * 2);
        vis_hi[mt] = cut_position(from + i);
        vis_lo[mt] = a.window ? cut_position(from + i - a.window + 1) : 0;
    }
    // ... and what all of them see
    const int all_hi = cut_position(from + token_of<true>(a, tile * ROWS)), all_lo = a.window ? cut_position(from + token_of<true>(a, tile * ROWS + rows - 1) - a.window + 1) : 0;
    __builtin_amdgcn_sched_barrier(0);
    if (begin < end) {
        const int page_v = there(pv, begin, grp);
        load_k(begin, there(pk, begin, col >> 2), true);
        pk = page_of(min(begin + 1, end - 1), col >> 2);
        pv = UNI ? pk : page_of(min(begin + 1, end - 1), grp);
        load_v(begin, page_v, true);
    }
    v4f o[MT][DT];
    float m[MT], l[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[mt][dt] = v4f{0.f, 0.f, 0.f, 0.f};
        m[mt] = M_NONE;
        l[mt] = 0.f;
        // the queries, requested first, have arrived before the loop: no wait for them inside it, which would be one for the codes
#pragma unroll
        for (int ks = 0; ks < 2 * KJ; ++ks) {
            v4i w = __builtin_bit_cast(v4i, qf[mt][ks]);
            asm volatile("" : "+v"(w));
            if (MT == 1) qf[mt][ks] = __builtin_bit_cast(v8bf, w);
            else qs[(mt * 2 * KJ + ks) * 64 + lane] = __builtin_bit_cast(v8bf, w);
        }
    }
    for (int j = begin; j < end; ++j) {
        // the codes of the next step are requested without a branch (what the compiler cannot count it waits for in full):
        // behind the last step, one address for all lanes
        const int next = min(j + 1, end - 1);
        const bool more = j + 1 < end;
        const int pos = range.position(j);
        const bool page_ok = (unsigned)v_page < c.page_limit;
        // ---- scores
        v4f s[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int t = 0; t < 4; ++t) s[mt][t] = v4f{0.f, 0.f, 0.f, 0.f};
        const float ksc = __int_as_float(k_scale << 23);
        int mine = lane;
        if constexpr (MT > 1) {
            asm volatile("" : "+v"(mine));                        // (so that they are not read once, before the loop, after all)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int ks = 0; ks < 2 * KJ; ++ks) qf[mt][ks] = qs[(mt * 2 * KJ + ks) * 64 + mine];
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int jj = 0; jj < KJ; ++jj)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const v8bf k = decode8<E5M2>(kr[t][jj][2 * e], kr[t][jj][2 * e + 1], ksc);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) s[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[mt][2 * jj + e], s[mt][t], 0, 0, 0);
                }
        // ---- the next step's keys, the pages of the one after it
        const int page_v = there(pv, next, grp);
        load_k(next, there(pk, next, col >> 2), more);
        pk = page_of(min(j + 2, end - 1), col >> 2);
        pv = UNI ? pk : page_of(min(j + 2, end - 1), grp);
        // ---- what is not seen
        const bool plain = pos + STEP - 1 <= all_hi && (pos >= all_lo || pos + STEP <= a.sinks) && __all(page_ok);
        float y[MT][16];                                          // position 16 grp + 4 t + r of the step at 4 t + r
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int e = 0; e < 16; ++e) y[mt][e] = s[mt][e >> 2][e & 3];
        if (!plain) {
            unsigned any = 0;
            const int base = pos + 16 * grp;
            auto below = [&](int at) { return (1u << min(max(at - base, 0), 16)) - 1u; };
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                // bit e: the lane's 16 positions
                const unsigned seen = page_ok ? below(vis_hi[mt] + 1) & (~below(vis_lo[mt]) | below(a.sinks)) : 0u;
                any |= seen;
#pragma unroll
                for (int e = 0; e < 16; ++e) y[mt][e] = (seen >> e) & 1u ? y[mt][e] : -INFINITY;
            }
            // over the rows: 16 columns hold different rows of the same positions
            any |= __builtin_amdgcn_mov_dpp(any, 0x121, 0xF, 0xF, true);
            any |= __builtin_amdgcn_mov_dpp(any, 0x122, 0xF, 0xF, true);
            any |= __builtin_amdgcn_mov_dpp(any, 0x124, 0xF, 0xF, true);
            any |= __builtin_amdgcn_mov_dpp(any, 0x128, 0xF, 0xF, true);
            // values that no row sees may be anything, the scale of their page too, and a NaN among the others must not reach the rows that do
            // not see it through a probability of zero: zeros instead, and NaN in the sums of those who see it
            if (!any) v_scale = 127;
            const unsigned limit = no_number_limit<E5M2>(v_scale);
            if (v_scale == 255) v_scale = 127;                    // (no code stays)
            bool bad = false;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int keep = bytes_of(any >> (4 * w));
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    vr[dt][w] &= keep;
                    const unsigned f = no_number((unsigned)vr[dt][w], limit);
                    if (f) bad = true;
                    vr[dt][w] &= (int)~((f >> 7) * 0xffu);
                }
            }
            if (__any(bad)) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const unsigned long long hit = nan_channels<D, E5M2>(a, b, h, pos, vis_lo[mt], vis_hi[mt], D / 4, [&](int i) { return (i >> 2) * 16 + 4 * grp + (i & 3); });
#pragma unroll
                    for (int i = 0; i < D / 4; ++i) o[mt][i >> 2][i & 3] = (hit >> i) & 1 ? NAN : o[mt][i >> 2][i & 3];
                }
            }
        }
        // ---- softmax: the maximum is looked for only where it was too low, which the sum of a lane's 16 probabilities shows (a sum of the
        // rounded ones, as the values' sums are)
        v8bf pf[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            int pw[8];
            float sum;
            auto probabilities = [&] {
                const float off = m[mt] * a.scale;
                const v2bf one = __builtin_bit_cast(v2bf, 0x3f803f80);
                float part[2] = {0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    pw[e] = pack_bf16(__builtin_amdgcn_exp2f(fmaf(y[mt][2 * e], a.scale, -off)), __builtin_amdgcn_exp2f(fmaf(y[mt][2 * e + 1], a.scale, -off)));
                    part[e & 1] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, pw[e]), one, part[e & 1], false);
                }
                sum = part[0] + part[1];
            };
            probabilities();
            if (__any(sum > 1024.f)) {
                float top = y[mt][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) top = fmaxf(top, y[mt][e]);
                const float up = fmaxf(m[mt], cross_group_max(top)), down = __builtin_amdgcn_exp2f((m[mt] - up) * a.scale);
                m[mt] = up;
                l[mt] *= down;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[mt][dt] *= down;
                probabilities();
            }
            l[mt] += sum;
            pf[mt][0] = __builtin_bit_cast(v8bf, v4i{pw[0], pw[1], pw[2], pw[3]});
            pf[mt][1] = __builtin_bit_cast(v8bf, v4i{pw[4], pw[5], pw[6], pw[7]});
        }
        // ---- values
        const float vsc = __int_as_float(v_scale << 23);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const v8bf v = decode8<E5M2>(vr[dt][2 * e], vr[dt][2 * e + 1], vsc);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) o[mt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[mt][e], o[mt][dt], 0, 0, 0);
            }
        load_v(next, page_v, more);
    }
    float* p = a.pieces + piece * x.piece_size;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const float sum = cross_group_sum(l[mt]);
        const int rr = mt * 16 + col;
        if (rr >= rows) continue;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) __builtin_nontemporal_store(o[mt][dt], (v4f*)(p + rr * D + dt * 16 + grp * 4));
        if (grp == 0) {
            p[x.piece_rows * D + rr] = m[mt];
            p[x.piece_rows * D + x.piece_rows + rr] = sum;
        }
    }
}

// Steps of a part at least.  Of a prefix (1, 2, 4, 8 steps), us: 32 sequences behind 4096 23.1, 23.3, 21.0, 26.2; 64 behind 1024 with parts of 2, 3, 4,
// 6: 22.8, 20.9, 22.2, 24.1.  Of a sequence's own (2, 4, 8), 64 in 16 groups 41.3, 40.3, 43.9; 256 behind 32768 210, 204, 208.
constexpr int MIN_MANY = 4, MIN_OWN = 4;
// What the sequences' own parts take of a CU's time beside a prefix's part, in steps of that: until a late part begins, and per step, for tiles of 16 and
// of 32 rows.  256 behind 32768 with half of them 210 us, with these 204, with twice as much 219.
constexpr float OWN_FIRST = 6.f, OWN_STEP[2] = {0.6f, 0.9f};
// Of the steps that two parts of prefixes do side by side on a CU, those of the one that began later (the SIMDs prefer older waves).  128 sequences behind
// 32768 with 0.375: the early ones end at 92 us, the late ones at 85; 0.42: 90 and 91; 0.5: 74 and 89.
constexpr float LATE = 0.42f;
// Steps of a late part at least: without late parts 256 behind 32768 take 239 us (204), 128 of one token behind 32768 116 (98); 1 or 8 instead of 3: the
// same within 1 % there.  64 of up to 512 behind 8192 have none by any of these, their own parts being counted as 11.9 steps beside 8 of the prefix: with a
// tenth to four tenths of the steps made late against that, 40 to 41 us instead of 33, and 32 under a window of 4096 37 to 38 instead of 35; each row then
// has twice the pieces to write and to join.
constexpr float MIN_LATE = 3.f;

// Rows of a sequence: tiles of 16 * MT.
template <int D, bool E5M2, int MT, bool UNI>
__global__ void __launch_bounds__(64 * WAVES, 2)
cache_shared_kernel(SharedArgs x)
{
    using Many = ManyLds<D>;
    constexpr int ROWS = 16 * MT, MANY = sizeof(typename Many::K) + sizeof(typename Many::V), Q = MT > 1 ? MT * (D / 32) * 64 : 1;
    static_assert(WAVES * Q * 16 <= MANY, "");
    __shared__ __attribute__((aligned(16))) char buffer[MANY];
    __shared__ int odd[4], some[4][WAVES], ends[5][WAVES], first[GROUPS_LDS + 1], steps[GROUPS_LDS];
    const CacheAttnArgs& a = x.a;
    const bool few_groups = x.g.n <= GROUPS_LDS;
    if (few_groups) {
        for (int g = threadIdx.x; g <= x.g.n; g += 64 * WAVES) first[g] = x.g.first[g];
        for (int g = threadIdx.x; g < x.g.n; g += 64 * WAVES) steps[g] = shared_steps(x, x.g.shared[g]);
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // ---- all there is to do: steps of the sequences' own, 256 sequences at a time, ...
    OwnSeq q4[4];
    auto load4 = [&](int base, bool wait) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int b = base + 64 * k + lane;
            const SeqInfo s = seq_of(a, min(b, a.s.B - 1));
            q4[k].start = s.start;
            q4[k].n = b < a.s.B ? s.n : 0;
        }
        if (wait) __syncthreads();                                // (the groups are in LDS)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int b = base + 64 * k + lane;
            q4[k].own = 0;
            if (base + 64 * k >= a.s.B) continue;                 // the same for all lanes
            const int g = few_groups ? group_of([&](int i) { return first[i]; }, x.g.n, b) : group_of([&](int i) { return x.g.first[i]; }, x.g.n, b);
            if (g >= 0) q4[k].own = few_groups ? steps[g] : shared_steps(x, x.g.shared[g]);
        }
    };
    constexpr bool ONE = MT == 1;                                 // a sequence's rows are one tile
    auto tiles_of = [&](const OwnSeq& q) { return ONE ? q.n > 0 : (int)(((unsigned)q.n * (unsigned)a.G + ROWS - 1) / ROWS); };
    float own_steps = 0.f;
    for (int base = 0; base < a.s.B; base += 256) {
        load4(base, base == 0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (base + 64 * k >= a.s.B) continue;
            const int n = tiles_of(q4[k]);
            for (int i = 0; i < n; ++i) own_steps += (float)own_range<ROWS, ONE>(a, q4[k], i).steps;
        }
    }
    own_steps = wave_sum(own_steps) * a.c.Hkv;
    // ... and of the groups' shared parts, 64 groups at a time
    Bounds r;
    int tiles, visited;
    auto load = [&](int g) {
        r = Bounds{0, 0, 0};
        if (g < x.g.n) {
            r.lo = min(max(few_groups ? first[g] : x.g.first[g], 0), a.s.B);
            r.hi = min(max(few_groups ? first[g + 1] : x.g.first[g + 1], r.lo), a.s.B);
            r.steps = few_groups ? steps[g] : shared_steps(x, x.g.shared[g]);
        }
        tiles = (int)(((unsigned)(r.hi - r.lo) * (unsigned)x.rows_per_seq + ROWS_MANY - 1) / ROWS_MANY);
        // under a window the steps differ from tile to tile: about as many as one token visits
        visited = a.window ? (int)min((int64_t)r.steps, (a.sinks + (int64_t)a.window + a.s.N) / STEP + 3) : r.steps;
    };
    float many = 0.f;
    for (int base = 0; base < x.g.n; base += 64) {
        load(base + lane);
        many += (float)tiles * (float)visited;
    }
    many = wave_sum(many) * a.c.Hkv;
    // ---- steps of a part
    auto part_of = [](float all, int parts, int least) {
        const float s = fminf(all / (float)parts, 1e9f);
        return max(__builtin_amdgcn_readfirstlane((int)ceilf(s)), least);
    };
    int share = part_of(many, x.cus, MIN_MANY);
    const int len = part_of(own_steps, x.more_own, MIN_OWN);
    auto pieces_of = [&] { return (int)min((int64_t)tiles * a.c.Hkv * ((visited + share - 1) / share), (int64_t)1 << 24); };
    auto count = [&] {
        int all = 0;
        for (int base = 0; base < x.g.n; base += 64) {
            if (x.g.n > 64) load(base + lane);
            all = max(all, 0) + __builtin_amdgcn_readlane(wave_scan(pieces_of()), 63);
        }
        return all;
    };
    int all = count();
    if (all > x.cus && all < 2 * x.cus) {                         // a few more than there are CUs: longer ones instead
        share = (int)((int64_t)share * all / x.cus) + 1;
        all = count();
    }
    // A CU holds two workgroups.  One takes the early steps of a prefix's part; the other takes sequences' own parts and, behind them, the part's late
    // steps, so many that both end together.
    const float each = many / (float)max(all, 1), own_time = OWN_FIRST + OWN_STEP[MT - 1] * own_steps / (float)x.cus;
    float early = 1.f;
    if (LATE * (each - own_time) > MIN_LATE) early = 1.f - LATE * (1.f - own_time / each);
    const bool two = early < 1.f;
    const int per = (all + 7) / 8;
    // ---- who does what, in the order of the workgroups
    int p = blockIdx.x;
    const bool late = p >= 8 * per;
    if (late) {
        // parts of what the sequences have to themselves, for each wave of its own: unit after unit in equal steps through all of them
        int units[4], upto[4], all_units = 0;
        auto count4 = [&](int base) {
            int sum = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                units[k] = upto[k] = 0;
                if (base + 64 * k >= a.s.B) continue;
                const int n = tiles_of(q4[k]);
                for (int i = 0; i < n; ++i) units[k] += max((own_range<ROWS, ONE>(a, q4[k], i).steps + len - 1) / len, 1);
                upto[k] = wave_scan(units[k]);
                sum += __builtin_amdgcn_readlane(upto[k], 63);
            }
            return sum * a.c.Hkv;
        };
        for (int base = 0; base < a.s.B; base += 256) {
            if (a.s.B > 256) load4(base, false);
            all_units += count4(base);
        }
        all_units = min(all_units, x.max_own);
        const int own_blocks = min((all_units + WAVES - 1) / WAVES, max(2 * x.cus - 8 * per, x.cus));
        p -= 8 * per;
        if (p < own_blocks) {
            // A wave's units only grow: each is looked for from the batch of sequences on that holds the one before it.  (From the first on, 16384
            // sequences of one token behind 512 took 9600 us.)
            int base = 0, before = 0;                             // the batch in the registers, and the units before it
            if (a.s.B > 256) {
                load4(base, false);
                count4(base);
            }
            for (int unit = p * WAVES + wave; unit < all_units; unit += own_blocks * WAVES) {
                int left = unit - before, b = -1, per_head = 1;
                OwnSeq sq = {0, 0, 0};
                for (;;) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (base + 64 * k >= a.s.B || b >= 0) continue;
                        const int sum = __builtin_amdgcn_readlane(upto[k], 63) * a.c.Hkv;
                        if (left >= sum) {
                            left -= sum;
                            continue;
                        }
                        const int who = __builtin_ctzll(__ballot(upto[k] * a.c.Hkv > left));
                        b = base + 64 * k + who;
                        sq.start = __builtin_amdgcn_readlane(q4[k].start, who);
                        sq.n = __builtin_amdgcn_readlane(q4[k].n, who);
                        sq.own = __builtin_amdgcn_readlane(q4[k].own, who);
                        per_head = __builtin_amdgcn_readlane(units[k], who);
                        left -= (__builtin_amdgcn_readlane(upto[k], who) - per_head) * a.c.Hkv;
                    }
                    if (b >= 0 || base + 256 >= a.s.B) break;
                    before = unit - left;
                    base += 256;
                    load4(base, false);
                    count4(base);
                }
                if (b < 0) break;
                const int h = left / per_head;
                int part = left - h * per_head, tile = 0, parts;
                OwnRange range;
                for (;; ++tile) {
                    range = own_range<ROWS, ONE>(a, sq, tile);
                    parts = max((range.steps + len - 1) / len, 1);
                    if (ONE || part < parts) break;
                    part -= parts;
                }
                if (part == 0 && lane == 0) {
                    const int64_t pair = (int64_t)b * a.c.Hkv + h;
                    a.split[pair * a.row_tiles + tile] = make_int2(unit, parts);
                    if (sq.own == 0) x.where[2 * pair] = make_int4(0, 0, 0, 0);
                }
                const int begin = (int)((int64_t)range.steps * part / parts), end = (int)((int64_t)range.steps * (part + 1) / parts);
                own_part<D, E5M2, MT, UNI>(x, sq, range, b, h, tile, begin, end, unit, (v8bf*)buffer + wave * Q);
            }
            __syncthreads();                                      // (the queries of every wave have been read)
        }
        // ... and behind them, or at once where there are none left, the late part of a prefix
        if (!two) return;
    }
    // a part of a prefix.  Workgroups next to each other in the list on the same XCD: they read the same keys
    const int at = p % 8 * per + p / 8;
    if (p >= 8 * per || at >= all) return;
    int before = 0;
    for (int base = 0; base < x.g.n; base += 64) {
        if (x.g.n > 64) load(base + lane);
        const int upto = wave_scan(pieces_of()), sum = __builtin_amdgcn_readlane(upto, 63);
        if (at >= before + sum) {
            before += sum;
            continue;
        }
        const int who = __builtin_ctzll(__ballot(before + upto > at));
        Bounds mine;
        mine.lo = __builtin_amdgcn_readlane(r.lo, who);
        mine.hi = __builtin_amdgcn_readlane(r.hi, who);
        mine.steps = __builtin_amdgcn_readlane(r.steps, who);
        const int n_tiles = __builtin_amdgcn_readlane(tiles, who), parts = (__builtin_amdgcn_readlane(visited, who) + share - 1) / share;
        const int first_piece = before + __builtin_amdgcn_readlane(upto, who) - n_tiles * a.c.Hkv * parts;
        const int i = at - first_piece, rest = i / n_tiles, tile = i - rest * n_tiles, h = rest / parts, part = rest - h * parts;
        const int item = h * n_tiles + tile;
        const int64_t piece = two ? 2 * ((int64_t)first_piece + item * parts + part) + late : (int64_t)first_piece + item * parts + part;
        if (i < 0 || h >= a.c.Hkv || piece < 0 || piece >= x.max_pieces) return;          // (bounds that decrease)
        const Many lds = {*(typename Many::K*)buffer, *(typename Many::V*)(buffer + sizeof(typename Many::K)), odd, some[0]};
        prefix_part<D, E5M2, UNI>(x, lds, ends, mine, h, tile, part, parts, early, late, piece, make_int2((first_piece + item * parts) << two, parts << two));
        return;
    }
}

// Joins the pieces of the prefix and of a sequence's own: a workgroup per sequence, kv head and 4 of its rows; threads over channels (4 each),
// rows and pieces, eight of a thread in flight.  64 sequences, 17 pieces of a row (19 MB): 6.5 us; 256 sequences, 9 to 10 (41 MB): 11.
template <int D, int ROWS, int T>
__global__ void __launch_bounds__(T)
cache_shared_join_kernel(SharedArgs x)
{
    constexpr int CH = D / 4, PG = T / (4 * CH), U = 8;
    const CacheAttnArgs& a = x.a;
    const int h = blockIdx.x % (unsigned)a.c.Hkv, b = blockIdx.x / (unsigned)a.c.Hkv;
    const int r0 = blockIdx.y * 4, rr = threadIdx.x / CH % 4, ch = threadIdx.x % CH, pg = threadIdx.x / (4 * CH);
    // ---- where the pieces are (within the workspace whatever the bounds of the groups say)
    const int64_t pair = (int64_t)b * a.c.Hkv + h;
    const SeqInfo sq = seq_of(a, b);
    const int4 in0 = x.where[2 * pair], in1 = x.where[2 * pair + 1];
    const int2 sp = a.split[pair * a.row_tiles + min(r0 + rr, x.rows_per_seq - 1) / ROWS];
    const int rows = sq.n * a.G;
    if (r0 >= rows) return;
    const int row = min(r0 + rr, rows - 1);
    const int4 in = row + in0.z < ROWS_MANY ? in0 : in1;
    const int own_first = max(sp.x, 0), own_n = (int)min((int64_t)max(sp.y, 0), max(x.max_own - own_first, (int64_t)0));
    const int many_first = max(in.x, 0), many_row = (row + in.z) & (ROWS_MANY - 1);
    const int many_n = in0.y == 0 ? 0 : (int)min((int64_t)max(in.y, 0), max(x.max_pieces - many_first, (int64_t)0));
    v4f o = {0.f, 0.f, 0.f, 0.f};
    float m = M_NONE, l = 0.f;
    const int n = own_n + many_n;
    for (int w = pg; w < n; w += PG * U) {
        float m2[U], l2[U];
        v4f y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = w + u * PG;
            m2[u] = M_NONE;
            l2[u] = 0.f;
            y[u] = v4f{0.f, 0.f, 0.f, 0.f};
            if (i < n) {
                const bool mine = i < own_n;
                const float* p = mine ? a.pieces + (int64_t)(own_first + i) * x.piece_size : x.pieces + (int64_t)(many_first + i - own_n) * (ROWS_MANY * (D + 2));
                const int at = mine ? row % ROWS : many_row, all = mine ? x.piece_rows : ROWS_MANY;
                m2[u] = p[all * D + at];
                l2[u] = p[all * D + all + at];
                y[u] = *(const v4f*)(p + at * D + ch * 4);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (w + u * PG >= n) break;
            const float up = fmaxf(m, m2[u]);
            const float f1 = __builtin_amdgcn_exp2f((m - up) * a.scale), f2 = __builtin_amdgcn_exp2f((m2[u] - up) * a.scale);
            m = up;
            l = l * f1 + l2[u] * f2;
            o = o * f1 + y[u] * f2;
        }
    }
    __shared__ v4f os[PG][4][CH];
    __shared__ float ms[PG][4], ls[PG][4];
    os[pg][rr][ch] = o;
    if (ch == 0) {
        ms[pg][rr] = m;
        ls[pg][rr] = l;
    }
    __syncthreads();
    if (pg || r0 + rr >= rows) return;
    for (int k = 1; k < min(PG, n); ++k) {
        const float m2 = ms[k][rr], up = fmaxf(m, m2);
        const float f1 = __builtin_amdgcn_exp2f((m - up) * a.scale), f2 = __builtin_amdgcn_exp2f((m2 - up) * a.scale);
        m = up;
        l = l * f1 + ls[k][rr] * f2;
        o = o * f1 + os[k][rr][ch] * f2;
    }
    const int i = row / a.G;
    char* op = a.out.data + b * a.out.stride_batch + (h * a.G + row - i * a.G) * a.out.stride_head + i * a.out.stride_token;
    const v4f y = o * (l == 0.f ? 0.f : 1.f / l);
    *(v2i*)(op + ch * 8) = v2i{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
}

// ---------------------------------------------------------------------------------------------------------------- host
// Sizes of a call: row tiles of a sequence, items of both kinds and their pieces at most.
struct SharedSizes {
    int mt, cus, more_own, piece_rows, piece_size;
    int64_t tiles, own_items, own_pieces, many_pieces, blocks;
    size_t bytes;
    bool fits;
};
static SharedSizes sizes_of(const CacheView& c, int B, int G, int N, int n_groups)
{
    SharedSizes z;
    const int64_t rows = (int64_t)N * G;
    z.mt = rows <= 16 ? 1 : 2;
    z.piece_rows = (int)std::min<int64_t>(rows, 16 * z.mt);
    z.piece_size = z.piece_rows * c.D + (2 * z.piece_rows + 3) / 4 * 4;
    z.tiles = (rows + 16 * z.mt - 1) / (16 * z.mt);
    z.cus = cache_cus();
    z.own_items = (int64_t)B * c.Hkv * z.tiles;
    z.more_own = (int)std::min<int64_t>(std::max<int64_t>(2 * z.own_items, 8 * z.cus), 16 * z.cus);
    z.own_pieces = z.more_own + z.own_items + 16;
    z.many_pieces = 2 * (z.cus + (B * rows / ROWS_MANY + std::min(n_groups, B) + 1) * (int64_t)c.Hkv);
    z.blocks = z.many_pieces + 32 + std::min<int64_t>((z.own_pieces + WAVES - 1) / WAVES, 2 * z.cus);
    z.bytes = (size_t)((z.own_pieces * z.piece_size + z.many_pieces * ROWS_MANY * (c.D + 2)) * 4 + (int64_t)B * c.Hkv * 32 + z.own_items * 8);
    z.fits = z.blocks * 256 <= 0xffffffffLL && (int64_t)B * c.Hkv * ((rows + 3) / 4) <= 0xffffffffLL / 512;
    return z;
}

// Whether sequences are taken together: where it saves reading this much once more, by the reach of the table (lengths are on the device), and
// the rows of one sequence do not fill half a tile anyway.  us together and by the kernels of dma_cache_attn, 32 query and 8 kv heads (MB repeated): 2
// behind 500 (1) 15.5, 9.0; 2 behind 8k (17) 20.7, 17.8; 8 behind 4096 (65) 21.6, 21.3; 32 behind 2000 (146) 21.5, 26.5; 64 behind 8k (1100) 34, 102.
// Under a table far wider than the sequences it chooses wrongly: 4 behind 1000 under one for 32768 16.6, 14.5 (by a table of their own width 10.7), 32 behind
// 300 18.9, 16.9.
// Rows of a sequence, 64 behind 8k: 16: 64, 107; 32: 100, 118; 64: 163, 262; 128: 320, 273.  More than 32 rows under a short table, where
// the other kernels read 128 rows' keys once as well: 170 random calls, geometric mean of the times' ratio: below 600 positions 2.0, to 1200 1.45, to 2500 1.1, to
// 5000 0.75, behind that 0.95 (up to 32 rows 0.54 to 1.05 everywhere).
constexpr int ROWS_TOGETHER = 64, ROWS_SHORT = 32, REACH_LONG = 2048;
constexpr double REPEATED = 1e8;
// Every workgroup goes through the batch and the groups to find its part: 5 ns of a call's time per workgroup and 256 sequences or 26 groups, but for the
// first 2500 of them, which run side by side.  The other kernels take 8 ns more per sequence and kv head.  Both as bytes that those would read
// again meanwhile, from the caches mostly (13 TB/s).  us together and by the other kernels, D = 128, one token: 4096 sequences behind 512 in one group, 8 kv
// heads of 4 query heads, 515, 980; in 1024 groups 5902, 1007; 16384 in one group, 1 kv head of 8, behind 4300 1611, 1654, behind 1000 1391, 639.  Of 612 calls
// of 200 to 16384 sequences in 1 to 2048 groups, 542 repeat 100 MB: 1.08 of the other kernels' time (geometric mean, 0.17 to 15.9); 139 of these are not taken
// together for this (2.5, 0.90 to 15.9), which leaves 0.81 (0.17 to 2.5; above 1.3 with few bytes of a sequence per kv head or 16 and 32 rows).
constexpr double FINDING = 8e4, FINDING_FREE = 2500, ITEM = 1e5, GROUP = 10;
static bool together(const SharedSizes& z, const CacheView& c, int B, int64_t rows, int n_groups, int window, int sinks)
{
    const int64_t capacity = (int64_t)c.max_pages << c.page_shift, reach = window ? std::min(capacity, (int64_t)window + sinks) : capacity;
    const double finding = FINDING * (z.blocks * (B + GROUP * n_groups) / 256 - FINDING_FREE) - ITEM * z.own_items;
    return n_groups > 0 && rows <= (reach >= REACH_LONG ? ROWS_TOGETHER : ROWS_SHORT) &&
           (double)(B - n_groups) * reach * 2 * c.Hkv * c.D >= REPEATED + std::max(finding, 0.0) && z.fits;
}

size_t cache_attn_shared_workspace(const CacheView& c, int B, int Hq, int N, int n_groups, int window, int sinks)
{
    const SharedSizes z = sizes_of(c, B, Hq / c.Hkv, N, n_groups);
    return together(z, c, B, (int64_t)N * (Hq / c.Hkv), n_groups, window, sinks) ? z.bytes : cache_attn_workspace(c, B, Hq, N, window, sinks);
}

template <int D, bool E5M2, int MT>
static int launch_shared(const SharedArgs& x, const SharedSizes& z, hipStream_t stream)
{
    const dim3 grid((unsigned)z.blocks), block(64 * WAVES);
    const int rc = x.a.c.page_shift >= 6 ? launch(cache_shared_kernel<D, E5M2, MT, true>, grid, block, stream, x) : launch(cache_shared_kernel<D, E5M2, MT, false>, grid, block, stream, x);
    if (rc != DMA_OK_) return rc;
    const dim3 join((unsigned)(x.a.s.B * x.a.c.Hkv), (unsigned)((x.rows_per_seq + 3) / 4));
    return (int64_t)join.x * join.y >= 4 * z.cus ? launch(cache_shared_join_kernel<D, 16 * MT, 256>, join, dim3(256), stream, x)
                                                 : launch(cache_shared_join_kernel<D, 16 * MT, 512>, join, dim3(512), stream, x);
}

int launch_cache_attn_shared(const CacheView& c, const Rows& q, const Rows& out, const Spans& s, int Hq, const Groups& groups, int window, int sinks,
                             void* workspace, hipStream_t stream)
{
    const SharedSizes z = sizes_of(c, s.B, Hq / c.Hkv, s.N, groups.n);
    if (!together(z, c, s.B, (int64_t)s.N * (Hq / c.Hkv), groups.n, window, sinks)) return launch_cache_attn(c, q, out, s, Hq, window, sinks, workspace, stream);
    SharedArgs x = {};
    CacheAttnArgs& a = x.a;
    a.c = c;
    a.q = q;
    a.out = out;
    a.s = s;
    a.G = Hq / c.Hkv;
    a.window = window;
    a.sinks = window ? sinks : 0;
    a.capacity = c.num_pages ? c.max_pages << c.page_shift : 0;
    a.scale = (float)(1.4426950408889634074 / sqrt((double)c.D));
    a.row_tiles = (int)z.tiles;
    x.g = groups;
    x.rows_per_seq = s.N * a.G;
    x.cus = z.cus;
    x.more_own = z.more_own;
    x.piece_rows = z.piece_rows;
    x.piece_size = z.piece_size;
    a.inv_g = (65536u + a.G - 1) / a.G;
    x.max_pieces = z.many_pieces;
    x.max_own = z.own_pieces;
    a.pieces = (float*)workspace;
    x.pieces = a.pieces + z.own_pieces * z.piece_size;
    x.where = (int4*)(x.pieces + z.many_pieces * ROWS_MANY * (c.D + 2));
    a.split = (int2*)(x.where + 2 * (int64_t)s.B * c.Hkv);
    auto pick = [&](auto D, auto F) { return z.mt == 1 ? launch_shared<D, F != 0, 1>(x, z, stream) : launch_shared<D, F != 0, 2>(x, z, stream); };
    if (c.D == 128) return c.e5m2 ? pick(IC<128>{}, IC<1>{}) : pick(IC<128>{}, IC<0>{});
    return c.e5m2 ? pick(IC<64>{}, IC<1>{}) : pick(IC<64>{}, IC<0>{});
}

}  // namespace dma
