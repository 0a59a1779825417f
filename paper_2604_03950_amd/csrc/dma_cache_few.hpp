// The steps of few query rows over the paged 8-bit cache (tiles of 16 * MT rows): of the sequences' whole contexts (dma_cache_attn.hip), or of
// what lies behind a prefix that they share (dma_cache_shared.hip).  What it does and measures is said at the first.
#pragma once

#include "dma_cache_device.hpp"
#include <math.h>

namespace dma {

constexpr int MIN_SHARE = 8;                 // steps (units): one or two for each wave

// What the waves share.  o: their sums; ml: maxima and weights; q: with 32 rows, the queries' operands, of which each wave loads some: in
// registers they would be spilled, and a reload waits for the codes in flight.  (Three arrays: as one object they cost registers, 16 spilled for 10.)
template <int D, int MT, int W>
struct FewLds {
    using O = float[W][16 * MT][D + 4];
    using Ml = float[W][2][16 * MT];
    using Q = v8bf[MT > 1 ? MT : 1][MT > 1 ? D / 32 : 1][MT > 1 ? 64 : 1];
    O& o;
    Ml& ml;
    Q& q;
};

// Sequences that share nothing: all of their steps are their own.
struct OwnAll {
    static constexpr bool ON = false;
    DMA_DEV SeqInfo seq(const CacheAttnArgs& a, int b) const { return seq_of(a, b); }
};

// BY_ITEM: one workgroup per item.  Otherwise the items' steps in equal shares.
// UNI: pages of 64 positions and more, so that a step lies in one: its page is the same for all lanes.
// own: the sequences and which of their steps are visited; where it leaves some out (ON), every item's sums go to the workspace.
// role(units of all items, block, blocks): which of the workgroups of the line this one is; false: none.
template <int D, bool E5M2, int MT, int W, bool BY_ITEM, bool UNI, typename Own, typename Role>
DMA_DEV void few_rows(const CacheAttnArgs& a, const FewLds<D, MT, W>& lds, const Own& own, Role&& role)
{
    constexpr int ROWS = 16 * MT, KJ = D / 64, DT = D / 16;
    constexpr bool ONE = MT == 1;            // a sequence's rows are one tile
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    const CacheView& c = a.c;
    const int page_mask = (1 << c.page_shift) - 1;

    // ---- where this workgroup's share lies: every wave finds it by itself, 256 sequences at a time
    int left = 1;                            // units of the share that are left
    int b = 0, h = 0, tile = 0;
    SeqInfo sq;
    int skip = 0;                            // steps of the first item that belong to others
    int wg = 0;                              // place in the line
    // units of an item
    auto units_of = [&](const SeqInfo& q, int i) { return (max(range_of<ROWS, ONE, Own::ON>(a, q, i).steps, 1) + (1 << a.unit_shift) - 1) >> a.unit_shift; };
    auto tiles_of = [&](const SeqInfo& q) { return ONE ? (q.n > 0) : (int)(((unsigned)q.n * (unsigned)a.G + ROWS - 1) / ROWS); };
    if constexpr (BY_ITEM) {
        unsigned i = blockIdx.x;
        if constexpr (!ONE) {
            tile = i % (unsigned)a.row_tiles;
            i /= (unsigned)a.row_tiles;
        }
        h = i % (unsigned)c.Hkv;
        b = i / (unsigned)c.Hkv;
        sq = own.seq(a, b);
        if (tile >= tiles_of(sq)) return;
    } else {
        SeqInfo q4[4];
        int mine[4], upto[4];                // units of a kv head of a lane's sequence, and of it and those before it among the 64
        auto load4 = [&](int first) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int bb = first + 64 * k + lane;
                q4[k] = own.seq(a, min(bb, a.s.B - 1));
                if (bb >= a.s.B) q4[k].n = 0;
            }
            int sum = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                mine[k] = 0;
                upto[k] = 0;
                if (first + 64 * k >= a.s.B) continue;                    // the same for all lanes
                const int tiles = tiles_of(q4[k]);
                for (int i = 0; i < tiles; ++i) mine[k] += units_of(q4[k], i);
                int x = mine[k];
                x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);       // row_shr:1, 2, 4, 8
                x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
                x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
                x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
                x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);       // row_bcast:15, 31
                x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
                upto[k] = x;
                sum += __builtin_amdgcn_readlane(x, 63);
            }
            return sum;
        };
        int total = 0;
        for (int first = 0; first < a.s.B; first += 256) total += load4(first);
        total *= c.Hkv;
        unsigned block, blocks;
        if (!role(total, block, blocks)) return;
        // one workgroup of four waves per CU instead of two where a share would be short: fewer pieces and starts (7 sequences of 0.6k-3k, 32
        // heads: 27.9 us with 512 shares of 14 steps, 30.9 with 420 of 16)
        int share = (int)(((unsigned)total + blocks - 1) / blocks);
        if (W == 4 && share < 10) share = (int)(((unsigned)total + blocks / 2 - 1) / (blocks / 2));
        share = max(share, MIN_SHARE);
        // workgroups next to each other in the line on the same XCD (they are dealt out in turn): they may share a sequence's keys
        const int shares = (int)(((unsigned)total + share - 1) / (unsigned)share), per = (shares + 7) / 8;
        wg = block % 8 * per + block / 8;
        if ((int)(block / 8) >= per || wg >= shares) return;
        int at = share * wg;
        left = min(share, total - at);
        // the sequence that holds the share's first unit
        for (int first = 0;; first += 256) {
            if (a.s.B > 256) load4(first);                                // (few: they are in the registers)
            bool found = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (found || first + 64 * k >= a.s.B) continue;
                const int all = __builtin_amdgcn_readlane(upto[k], 63) * c.Hkv;
                if (at < all) {
                    const int who = __builtin_ctzll(__ballot(upto[k] * c.Hkv > at));
                    b = first + 64 * k + who;
                    sq.start = __builtin_amdgcn_readlane(q4[k].start, who);
                    sq.n = __builtin_amdgcn_readlane(q4[k].n, who);
                    if constexpr (Own::ON) sq.own = __builtin_amdgcn_readlane(q4[k].own, who);
                    const int per_head = __builtin_amdgcn_readlane(mine[k], who);
                    at -= (__builtin_amdgcn_readlane(upto[k], who) - per_head) * c.Hkv;
                    h = (int)((unsigned)at / (unsigned)per_head);
                    at -= h * per_head;
                    found = true;
                } else {
                    at -= all;
                }
            }
            if (found) break;
        }
        if constexpr (!ONE) {
            for (;; ++tile) {
                const int w = units_of(sq, tile);
                if (at < w) break;
                at -= w;
            }
        }
        skip = at << a.unit_shift;
    }

    // ---- item after item.  The codes of an item's first steps are requested before the sums of the one before it are joined.
    StepRange range = {0, 0, 0};
    int weight = 1, until = 0, rows = 0, all_hi = 0, all_lo = 0, last = 0, j = 0;
    v8bf qf[MT == 1 ? 2 * KJ : (MT * 2 * KJ + W - 1) / W];
    int vis_lo[MT], vis_hi[MT];              // what the row of this lane's column sees: these positions and those below sinks
    const int* table = nullptr;
    v4i kr[4][KJ], vr[DT];
    uint8_t k_scale = 0, v_scale = 0;
    int v_page = -1, pk = -1, pv = -1;       // pages of the step after the next
    // Pages of a step: of the 16 positions whose keys this lane loads, and of those whose values it loads.  Requested a step ahead, and
    // looked at (behind the table: no page) only where they are used: looking at once would wait for the codes too.
    auto page_of = [&](int jj, int g) -> int {
        const int at = min((range.position(jj) + (UNI ? 0 : 16 * g)) >> c.page_shift, c.max_pages - 1);
        return UNI ? scalar_at(table, __builtin_amdgcn_readfirstlane(at)) : table[at];
    };
    auto there = [&](int page, int jj, int g) -> int {
        if constexpr (!UNI) asm volatile("" : "+v"(page));
        return (range.position(jj) + (UNI ? 0 : 16 * g)) >> c.page_shift < c.max_pages ? page : -1;
    };
    auto slab_of = [&](int page) -> int64_t {
        if constexpr (UNI) page = __builtin_amdgcn_readfirstlane(page);
        return (int64_t)((unsigned)page < c.page_limit ? page : 0) * c.Hkv + h;
    };
    // the positions of a lane's keys: 16 (col / 4) + 4 t + col % 4 in product t
    auto load_k = [&](int jj, int page, bool on) {
        const int64_t slab = slab_of(page);
        const int pos = range.position(jj), at = 16 * (col >> 2);
        const uint8_t* base = c.k_codes + ((slab << c.page_shift) + ((UNI ? pos : pos + at) & page_mask)) * D;
        const uint8_t* p = base + (on ? (unsigned)(((UNI ? at : 0) + (col & 3)) * D + grp * 16) : 0u);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < KJ; ++i) kr[t][i] = *(const v4i*)(p + t * 4 * D + i * 64);
        k_scale = c.k_scales[slab];
    };
    auto load_v = [&](int jj, int page, bool on) {
        const int64_t slab = slab_of(page);
        const int pos = range.position(jj);
        const uint8_t* base = c.v_codes + ((slab * D) << c.page_shift) + ((UNI ? pos : pos + 16 * grp) & page_mask);
        const unsigned mine = on ? (col << c.page_shift) + (UNI ? 16 * grp : 0) : 0u;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vr[dt] = *(const v4i*)(base + ((dt * 16) << c.page_shift) + mine);
        v_scale = c.v_scales[slab];
        v_page = page;
    };

    v4f o[MT][DT];
    float m[MT], l[MT];
    int old_b = 0, old_h = 0, old_tile = 0, old_rows = 0, old_piece = 0;      // the item whose sums are in o; its piece: -1: all of it
    bool more = true;
    for (;;) {
        if (more) {
            range = range_of<ROWS, ONE, Own::ON>(a, sq, tile);
            weight = max(range.steps, 1);
            until = BY_ITEM ? weight : (int)min((int64_t)weight, skip + ((int64_t)left << a.unit_shift));
            rows = min(sq.n * a.G - tile * ROWS, ROWS);
            last = min(until, range.steps);
            j = skip + wave;
            table = c.page_table + (int64_t)b * c.max_pages;
            if (j < last) {
                pk = page_of(j, col >> 2);
                pv = UNI ? pk : page_of(j, grp);
            }
            const int64_t from = sq.start;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int r = min(mt * 16 + col, rows - 1) + tile * ROWS, i = token_of<ONE>(a, r);
                const char* qp = a.q.data + b * a.q.stride_batch + (h * a.G + r - i * a.G) * a.q.stride_head + i * a.q.stride_token;
#pragma unroll
                for (int ks = 0; ks < 2 * KJ; ++ks)
                    if (MT == 1) qf[ks] = *(const v8bf*)(qp + ((ks >> 1) * 64 + grp * 16 + (ks & 1) * 8) * 2);
                    else if ((mt * 2 * KJ + ks) % W == wave) qf[(mt * 2 * KJ + ks) / W] = *(const v8bf*)(qp + ((ks >> 1) * 64 + grp * 16 + (ks & 1) * 8) * 2);
                vis_hi[mt] = (int)min(from + i, (int64_t)POS_MAX);
                vis_lo[mt] = a.window ? (int)min(max(from + i - a.window + 1, (int64_t)0), (int64_t)POS_MAX) : 0;
            }
            // ... and what all of them see
            all_hi = (int)min(from + (ONE ? 0 : tile * ROWS / a.G), (int64_t)POS_MAX);
            all_lo = a.window ? (int)min(max(from + token_of<ONE>(a, tile * ROWS + rows - 1) - a.window + 1, (int64_t)0), (int64_t)POS_MAX) : 0;
            __builtin_amdgcn_sched_barrier(0);
            if (j < last) {
                const int page_v = there(pv, j, grp);
                load_k(j, there(pk, j, col >> 2), true);
                pk = page_of(min(j + W, last - 1), col >> 2);
                pv = UNI ? pk : page_of(min(j + W, last - 1), grp);
                load_v(j, page_v, true);
            }
        }

        // ---- the sums of the waves: of the item before
        if (old_rows) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const float sum = cross_group_sum(l[mt]);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) *(v4f*)&lds.o[wave][mt * 16 + col][dt * 16 + grp * 4] = o[mt][dt];
                if (grp == 0) {
                    lds.ml[wave][0][mt * 16 + col] = m[mt];
                    lds.ml[wave][1][mt * 16 + col] = sum;
                }
            }
            __syncthreads();
            for (int at = threadIdx.x; at < old_rows * (D / 4); at += 64 * W) {
                const int rr = at / (D / 4), ch = at % (D / 4);
                float up = M_NONE, sum = 0.f;
                for (int w = 0; w < W; ++w) up = fmaxf(up, lds.ml[w][0][rr]);
                v4f x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float f = __builtin_amdgcn_exp2f((lds.ml[w][0][rr] - up) * a.scale);
                    sum += lds.ml[w][1][rr] * f;
                    x += *(const v4f*)&lds.o[w][rr][ch * 4] * f;
                }
                if (BY_ITEM || old_piece < 0) {
                    const int r = old_tile * ROWS + rr, i = token_of<ONE>(a, r);
                    char* op = a.out.data + old_b * a.out.stride_batch + (old_h * a.G + r - i * a.G) * a.out.stride_head + i * a.out.stride_token;
                    x *= sum == 0.f ? 0.f : 1.f / sum;
                    *(v2i*)(op + ch * 8) = v2i{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
                } else {
                    float* p = a.pieces + (int64_t)old_piece * (ROWS * (D + 2));
                    *(v4f*)(p + rr * D + ch * 4) = x;
                    if (ch == 0) {
                        p[ROWS * D + rr] = up;
                        p[ROWS * D + ROWS + rr] = sum;
                    }
                }
            }
            if (!more) return;
            if constexpr (MT == 1) __syncthreads();               // before the next item's sums
        }
        if constexpr (MT > 1) {
#pragma unroll
            for (int f = 0; f < MT * 2 * KJ; ++f)
                if (f % W == wave) lds.q[f / (2 * KJ)][f % (2 * KJ)][lane] = qf[f / W];
            __syncthreads();
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[mt][dt] = v4f{0.f, 0.f, 0.f, 0.f};
            m[mt] = M_NONE;
            l[mt] = 0.f;
        }
        // the queries, requested first, have arrived before the loop: no wait for them inside it, which would be one for the codes
        if constexpr (MT == 1) {
#pragma unroll
            for (int ks = 0; ks < 2 * KJ; ++ks) {
                v4i w = __builtin_bit_cast(v4i, qf[ks]);
                asm volatile("" : "+v"(w));
                qf[ks] = __builtin_bit_cast(v8bf, w);
            }
        }
        for (; j < last; j += W) {
            // the codes of the next step are requested without a branch (what the compiler cannot count it waits for in full):
            // behind the last step, one address for all lanes
            const int next = min(j + W, last - 1);
            const bool more = j + W < last;
            const int pos = range.position(j);
            const bool page_ok = (unsigned)v_page < c.page_limit;
            // ---- scores
            v4f s[MT][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int t = 0; t < 4; ++t) s[mt][t] = v4f{0.f, 0.f, 0.f, 0.f};
            const float ksc = __int_as_float(k_scale << 23);
            v8bf qk[MT][2 * KJ];
            int mine = lane;
            if constexpr (MT > 1) asm volatile("" : "+v"(mine));  // (so that they are not read once, before the loop, after all)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int ks = 0; ks < 2 * KJ; ++ks) qk[mt][ks] = MT == 1 ? qf[ks] : lds.q[MT > 1 ? mt : 0][MT > 1 ? ks : 0][MT > 1 ? mine : 0];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int jj = 0; jj < KJ; ++jj)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const v8bf k = decode8<E5M2>(kr[t][jj][2 * e], kr[t][jj][2 * e + 1], ksc);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) s[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qk[mt][2 * jj + e], s[mt][t], 0, 0, 0);
                    }
            // ---- the next step's keys, the pages of the one after it
            const int page_v = there(pv, next, grp);
            load_k(next, there(pk, next, col >> 2), more);
            pk = page_of(min(j + 2 * W, last - 1), col >> 2);
            pv = UNI ? pk : page_of(min(j + 2 * W, last - 1), grp);
            // ---- what is not seen
            const bool plain = pos + STEP - 1 <= all_hi && (pos >= all_lo || pos + STEP <= a.sinks) && __all(page_ok);
            float x[MT][16];                                      // position 16 grp + 4 t + r of the step at 4 t + r
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int e = 0; e < 16; ++e) x[mt][e] = s[mt][e >> 2][e & 3];
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
                    for (int e = 0; e < 16; ++e) x[mt][e] = (seen >> e) & 1u ? x[mt][e] : -INFINITY;
                }
                // over the rows: 16 columns hold different rows of the same positions
                any |= __builtin_amdgcn_mov_dpp(any, 0x121, 0xF, 0xF, true);
                any |= __builtin_amdgcn_mov_dpp(any, 0x122, 0xF, 0xF, true);
                any |= __builtin_amdgcn_mov_dpp(any, 0x124, 0xF, 0xF, true);
                any |= __builtin_amdgcn_mov_dpp(any, 0x128, 0xF, 0xF, true);
                // values that no row sees may be anything, and a NaN among the others must not reach the rows that do not see it
                // through a probability of zero: zeros instead, and NaN in the sums of those who see it.  Nor may the scale of a page of which
                // no row sees anything, or of page 0 in the place of none: with 255 a zero is decoded to NaN
                if (!any) v_scale = 127;
                bool bad = false;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int keep = bytes_of(any >> (4 * w));
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        vr[dt][w] &= keep;
                        const unsigned f = no_number<E5M2>((unsigned)vr[dt][w]);
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
            // ---- softmax
            v8bf pf[MT][2];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                // the maximum is looked for only where it was too low: the sum of a lane's 16 probabilities shows it (and is a sum of
                // the rounded ones, as the values' sums are)
                int pw[8];
                float sum;
                auto probabilities = [&] {
                    const float off = m[mt] * a.scale;
                    const v2bf one = __builtin_bit_cast(v2bf, 0x3f803f80);
                    float part[2] = {0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        pw[e] = pack_bf16(__builtin_amdgcn_exp2f(fmaf(x[mt][2 * e], a.scale, -off)), __builtin_amdgcn_exp2f(fmaf(x[mt][2 * e + 1], a.scale, -off)));
                        part[e & 1] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, pw[e]), one, part[e & 1], false);
                    }
                    sum = part[0] + part[1];
                };
                probabilities();
                if (__any(sum > 1024.f)) {
                    float top = x[mt][0];
#pragma unroll
                    for (int e = 1; e < 16; ++e) top = fmaxf(top, x[mt][e]);
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

        // ---- what was worked on, and what comes next
        old_b = b;
        old_h = h;
        old_tile = tile;
        old_rows = rows;
        if constexpr (BY_ITEM) more = false;
        else {
            const bool first = skip == 0, ends = until == weight;
            const int64_t item = ((int64_t)b * c.Hkv + h) * a.row_tiles + tile;
            if constexpr (Own::ON) old_piece = wg + (int)item;     // all are joined: one more with every workgroup and every item
            else old_piece = first && ends ? -1 : 2 * wg + first;
            if (threadIdx.x == 0) {
                int* sp = (int*)(a.split + item);
                const int name = Own::ON ? old_piece : wg;
                if (first) sp[0] = name;                           // the first piece's workgroup says so ...
                if (ends) sp[1] = name;                            // ... and the last one's
            }
            left -= (until - skip + (1 << a.unit_shift) - 1) >> a.unit_shift;
            skip = 0;
            more = left > 0;
            if (more) {
                ++tile;
                while (tile >= tiles_of(sq)) {
                    tile = 0;
                    if (h + 1 < c.Hkv && sq.n > 0) ++h;
                    else {
                        h = 0;
                        sq = own.seq(a, ++b);
                    }
                }
            }
        }
    }
}

}  // namespace dma
