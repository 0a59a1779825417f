// Attention over the paged 8-bit cache for few query rows per kv head (single tokens, drafts): bound by the bytes of the cache.
//
// Rows: the query tokens of a sequence times the G query heads of a kv head, token by token, in tiles of 16 * MT.  A step is 64
// positions.  A wave forms S^T = K Q^T with the matrix instruction's 16 rows set to positions such that lane group g (16 lanes) of
// the result holds positions 16 g .. 16 g + 15 of the step, 4 per product: exactly the ones whose probabilities that group has to
// give to O^T = V^T P^T, so P never leaves its lane, and each operand of V is 16 consecutive bytes of the cache (its positions lie
// innermost).  Codes go from memory to registers once and are decoded to bf16 there, times the page's scale (exact); no LDS until
// the waves of a workgroup, which take turns at the steps, join their sums.
//
// Softmax: base 2, one maximum per row, raised only where it was far too low (then everything is scaled down): p <= 2^10, and a step
// needs no exchange between lanes.  bf16's rounding of p is relative and does not notice; the sums of n keys stay below 2^7 (n + 64) max|v|
// (16 positions of a lane have p of 1024 together at most), in binary32 for every value below 2^121 / (n + 64).
//
// p is rounded to bf16 because the matrix instruction takes both operands in one type, and bf16 is the one that decoded values fit without
// rounding (their exponents do not fit binary16).  It costs 2^-8 of the weighted mean of |v| and |o| at most; over 1k to 32k keys the results
// are 0.0017 to 0.0021 from those in 64 bits (relative, over all elements), with unrounded p 0.0016 to 0.0017: their own rounding to bf16.  p in two
// bf16 terms would take the second product twice.
//
// Long and uneven sequences: the steps of all (sequence, kv head, row tile) items form one line that is cut into equal shares, one
// per workgroup.  An item that lies in one share is written directly; pieces of the others go to the workspace, and a second
// kernel joins them.  Where no item is long, a workgroup per item and no second kernel.
//
// Measured (a copy of 201 MB runs at 6.2 TB/s here), 32 query and 8 kv heads, D = 128, E4M3, pages of 64, one token per sequence: 64 sequences
// of up to 8k (599 MB of codes) 111 us = 5.4 TB/s, and 4.7 us for the join; one of 32k (67 MB) 15.6 us = 4.3 TB/s, and 3.9; one of 1k (2 MB)
// 10.5 us, in one kernel.  The loop itself runs at about 6.2 TB/s; the rest is a start of 5 us (page table, codes and queries arrive one after
// the other), the join, and shares that end unevenly.
#include "dma_cache_device.hpp"
#include <algorithm>
#include <atomic>
#include <math.h>

namespace dma {

constexpr int MIN_SHARE = 8;                 // steps (units): one or two for each wave

// BY_ITEM: one workgroup per item.  Otherwise the items' steps in equal shares.
// UNI: pages of 64 positions and more, so that a step lies in one: its page is the same for all lanes.
template <int D, bool E5M2, int MT, int W, bool BY_ITEM, bool UNI>
__global__ void __launch_bounds__(64 * W, 2)
cache_attn_kernel(CacheAttnArgs a)
{
    constexpr int ROWS = 16 * MT, KJ = D / 64, DT = D / 16, LD = D + 4;
    constexpr bool ONE = MT == 1;            // a sequence's rows are one tile
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    __shared__ __attribute__((aligned(16))) float obuf[W][ROWS][LD];
    __shared__ float ml[W][2][ROWS];
    // with 32 rows, the queries' operands, of which each wave loads some: in registers they would be spilled, and a reload waits for the codes in flight
    __shared__ __attribute__((aligned(16))) v8bf qs[MT > 1 ? MT : 1][MT > 1 ? 2 * KJ : 1][MT > 1 ? 64 : 1];
    const CacheView& c = a.c;
    const int page_mask = (1 << c.page_shift) - 1;

    // ---- where this workgroup's share lies: every wave finds it by itself, 256 sequences at a time
    int left = 1;                            // units of the share that are left
    int b = 0, h = 0, tile = 0;
    SeqInfo sq;
    int skip = 0;                            // steps of the first item that belong to others
    int wg = 0;                              // place in the line
    // units of an item
    auto units_of = [&](const SeqInfo& q, int i) { return (max(range_of<ROWS, ONE>(a, q, i).steps, 1) + (1 << a.unit_shift) - 1) >> a.unit_shift; };
    auto tiles_of = [&](const SeqInfo& q) { return ONE ? (q.n > 0) : (int)(((unsigned)q.n * (unsigned)a.G + ROWS - 1) / ROWS); };
    if constexpr (BY_ITEM) {
        unsigned i = blockIdx.x;
        if constexpr (!ONE) {
            tile = i % (unsigned)a.row_tiles;
            i /= (unsigned)a.row_tiles;
        }
        h = i % (unsigned)c.Hkv;
        b = i / (unsigned)c.Hkv;
        sq = seq_of(a, b);
        if (tile >= tiles_of(sq)) return;
    } else {
        SeqInfo q4[4];
        int mine[4], upto[4];                // units of a kv head of a lane's sequence, and of it and those before it among the 64
        auto load4 = [&](int first) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int bb = first + 64 * k + lane;
                q4[k] = seq_of(a, min(bb, a.s.B - 1));
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
        // one workgroup of four waves per CU instead of two where a share would be short: fewer pieces and starts (7 sequences of 0.6k-3k, 32
        // heads: 27.9 us with 512 shares of 14 steps, 30.9 with 420 of 16)
        int share = (int)(((unsigned)total + gridDim.x - 1) / gridDim.x);
        if (W == 4 && share < 10) share = (int)(((unsigned)total + gridDim.x / 2 - 1) / (gridDim.x / 2));
        share = max(share, MIN_SHARE);
        // workgroups next to each other in the line on the same XCD (they are dealt out in turn): they may share a sequence's keys
        const int shares = (int)(((unsigned)total + share - 1) / (unsigned)share), per = (shares + 7) / 8;
        wg = blockIdx.x % 8 * per + blockIdx.x / 8;
        if ((int)(blockIdx.x / 8) >= per || wg >= shares) return;
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
            range = range_of<ROWS, ONE>(a, sq, tile);
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
                for (int dt = 0; dt < DT; ++dt) *(v4f*)&obuf[wave][mt * 16 + col][dt * 16 + grp * 4] = o[mt][dt];
                if (grp == 0) {
                    ml[wave][0][mt * 16 + col] = m[mt];
                    ml[wave][1][mt * 16 + col] = sum;
                }
            }
            __syncthreads();
            for (int at = threadIdx.x; at < old_rows * (D / 4); at += 64 * W) {
                const int rr = at / (D / 4), ch = at % (D / 4);
                float up = M_NONE, sum = 0.f;
                for (int w = 0; w < W; ++w) up = fmaxf(up, ml[w][0][rr]);
                v4f x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float f = __builtin_amdgcn_exp2f((ml[w][0][rr] - up) * a.scale);
                    sum += ml[w][1][rr] * f;
                    x += *(const v4f*)&obuf[w][rr][ch * 4] * f;
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
                if (f % W == wave) qs[f / (2 * KJ)][f % (2 * KJ)][lane] = qf[f / W];
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
                for (int ks = 0; ks < 2 * KJ; ++ks) qk[mt][ks] = MT == 1 ? qf[ks] : qs[MT > 1 ? mt : 0][MT > 1 ? ks : 0][MT > 1 ? mine : 0];
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
            old_piece = first && ends ? -1 : 2 * wg + first;
            if (threadIdx.x == 0) {
                int* sp = (int*)(a.split + ((int64_t)b * c.Hkv + h) * a.row_tiles + tile);
                if (first) sp[0] = wg;                             // the first piece's workgroup says so ...
                if (ends) sp[1] = wg;                              // ... and the last one's
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
                        sq = seq_of(a, ++b);
                    }
                }
            }
        }
    }
}

// Joins the pieces of split items: a workgroup per item and 4 of its rows; threads over channels (4 each), rows and pieces,
// a thread's loads of several pieces in flight at a time.  Bound by latency: three dependent loads.
template <int D, int ROWS>
__global__ void __launch_bounds__(1024)
cache_attn_join_kernel(CacheAttnArgs a)
{
    constexpr int CH = D / 4, PG = 1024 / (4 * CH), U = 4;
    unsigned item = blockIdx.x;
    const int tile = item % (unsigned)a.row_tiles;
    const int h = item / (unsigned)a.row_tiles % (unsigned)a.c.Hkv, b = item / (unsigned)a.row_tiles / (unsigned)a.c.Hkv;
    const int2 sp = a.split[item];                              // anything where the item does not exist
    const SeqInfo sq = seq_of(a, b);
    const int rows = (int)min((int64_t)sq.n * a.G - (int64_t)tile * ROWS, (int64_t)ROWS);
    const int rr = blockIdx.y * 4 + threadIdx.x / CH % 4, ch = threadIdx.x % CH, pg = threadIdx.x / (4 * CH);
    if ((int)blockIdx.y * 4 >= rows || sp.x == sp.y) return;
    __shared__ v4f os[PG][4][CH];
    __shared__ float ms[PG][4], ls[PG][4];
    v4f o = {0.f, 0.f, 0.f, 0.f};
    float m = M_NONE, l = 0.f;
    const int r0 = min(rr, rows - 1);
    for (int w = sp.x + pg; w <= sp.y; w += PG * U) {
        float m2[U], l2[U];
        v4f x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int wu = w + u * PG;
            m2[u] = M_NONE;
            l2[u] = 0.f;
            x[u] = v4f{0.f, 0.f, 0.f, 0.f};
            if (wu <= sp.y) {
                const float* p = a.pieces + (int64_t)(2 * wu + (wu == sp.x)) * (ROWS * (D + 2));
                m2[u] = p[ROWS * D + r0];
                l2[u] = p[ROWS * D + ROWS + r0];
                x[u] = *(const v4f*)(p + r0 * D + ch * 4);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (w + u * PG > sp.y) break;
            const float up = fmaxf(m, m2[u]);
            const float f1 = __builtin_amdgcn_exp2f((m - up) * a.scale), f2 = __builtin_amdgcn_exp2f((m2[u] - up) * a.scale);
            m = up;
            l = l * f1 + l2[u] * f2;
            o = o * f1 + x[u] * f2;
        }
    }
    os[pg][rr & 3][ch] = o;
    if (ch == 0) {
        ms[pg][rr & 3] = m;
        ls[pg][rr & 3] = l;
    }
    __syncthreads();
    if (pg || rr >= rows) return;
    const int groups = min(PG, sp.y - sp.x + 1);
    for (int k = 1; k < groups; ++k) {
        const float m2 = ms[k][rr & 3], up = fmaxf(m, m2);
        const float f1 = __builtin_amdgcn_exp2f((m - up) * a.scale), f2 = __builtin_amdgcn_exp2f((m2 - up) * a.scale);
        m = up;
        l = l * f1 + ls[k][rr & 3] * f2;
        o = o * f1 + os[k][rr & 3][ch] * f2;
    }
    const int r = tile * ROWS + rr, i = r / a.G;
    char* op = a.out.data + b * a.out.stride_batch + (h * a.G + r - i * a.G) * a.out.stride_head + i * a.out.stride_token;
    const v4f x = o * (l == 0.f ? 0.f : 1.f / l);
    *(v2i*)(op + ch * 8) = v2i{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
}

// ---------------------------------------------------------------------------------------------------------------- host
int cache_cus()
{
    static std::atomic<int> cached[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    n = cached[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 256;
        cached[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

// Rows per workgroup: 16 where a kv head has no more, else 32.
static int mt_of(int G, int N) { return (int64_t)G * N <= 16 ? 1 : 2; }

// Waves of a workgroup where the steps are cut in shares; the chip holds 8 / waves of them per CU.  Eight where items are few: half the starts
// and pieces for the same bytes.  Four otherwise: the waves of a workgroup end an item together, so eight leave more of a CU idle at its
// end.  us with four and with eight, 16 rows: one sequence of 8k (8 items) 15.3, 13.2; of 128k 56.0, 53.8; 16 of 4k (128 items) 32.0, 31.6;
// 32 of 0.4k-4k (256 items) 37.1, 41.7; 64 of 16k (512 items) 358, 377; 32 rows: 16 of 4k x 16 tokens (256 items) 49.2, 44.0;
// 32 of 2k x 16 tokens (512 items) 52.0, 64.2.
static int waves_of(int mt, int64_t items) { return items <= (mt == 1 ? cache_cus() / 2 : cache_cus()) ? 8 : 4; }
// (A multiple of 8, for the order over the XCDs.)
static int64_t grid_of(int waves) { return ((int64_t)cache_cus() * 8 / waves + 7) / 8 * 8; }

// Whether the kernel for many rows serves the call: where the other one would need more than two tiles of 32 rows, and with two of them
// where sequences and kv heads alone give every CU an item of 128 rows.  us with the kernel for few and the one for many: 32 rows,
// 64 sequences of 0.4k-4k 92.8, 100; 64 rows: 16 of 4k (128 pairs) 44.0, 49.6; 32 of 2k (256) 52.2, 58.7; 64 of 0.4k-4k (512) 130, 114;
// 16 of 2k, 32 kv heads (512) 109, 77; D = 64, 64 of 2k (512) 65.1, 53.4; 80 rows: 16 of 4k 81.5, 53.0; one of 32k 42.4, 39.0.
static bool many_rows(int B, int Hkv, int G, int N)
{
    const int64_t rows = (int64_t)N * G;
    return rows > 64 || (rows > 32 && (int64_t)B * Hkv > cache_cus());
}

// The most positions that a row tile can visit.
static int64_t reach_of(const CacheView& c, int rows, int G, int window, int sinks)
{
    const int64_t capacity = (int64_t)c.max_pages << c.page_shift;
    return window ? std::min(capacity, (int64_t)window + std::min(sinks, 1 << 30) + rows / G + 3 * STEP) : capacity;
}
// One workgroup per item, eight waves of it, where no item is longer than this: a second kernel to join pieces costs more than the
// chip's other CUs save (one sequence of 1000, 8 kv heads: 10.0 us as one kernel, 11.8 with the shares and the join).  What counts is
// the reach of the table, as the lengths are on the device: under a table for 32k the sequence of 1000 takes the 11.8.
constexpr int64_t SHORT_REACH = 20 * STEP;

// Workgroups per item of the join, and whether a launch can hold the items' threads.
static int64_t join_groups(int rows, int G, int N) { return std::min<int64_t>(rows / 4, ((int64_t)N * G + 3) / 4); }
static bool few_fit(int64_t items, int64_t threads_per_item) { return items <= 0xffffffffLL / threads_per_item; }

size_t cache_attn_workspace(const CacheView& c, int B, int Hq, int N, int window, int sinks)
{
    const int G = Hq / c.Hkv;
    if (many_rows(B, c.Hkv, G, N)) return cache_prompt_workspace(B, c.Hkv, G, N, c.D, reach_of(c, 128, G, window, sinks));
    const int mt = mt_of(G, N), rows = 16 * mt;
    if (reach_of(c, rows, G, window, sinks) <= SHORT_REACH) return 0;
    const int64_t tiles = ((int64_t)N * G + rows - 1) / rows, items = (int64_t)B * c.Hkv * tiles;
    if (!few_fit(items, join_groups(rows, G, N) * 1024)) return 0;
    return (size_t)(2 * grid_of(waves_of(mt, items)) * rows * (c.D + 2) * 4 + items * 8);
}

template <int D, bool E5M2, int MT>
static int launch_few(CacheAttnArgs a, void* workspace, hipStream_t stream)
{
    constexpr int ROWS = 16 * MT;
    const int64_t tiles = ((int64_t)a.s.N * a.G + ROWS - 1) / ROWS, items = (int64_t)a.s.B * a.c.Hkv * tiles;
    a.row_tiles = (int)tiles;
    const bool uni = a.c.page_shift >= 6;
    if (reach_of(a.c, ROWS, a.G, a.window, a.sinks) <= SHORT_REACH) {
        if (!few_fit(items, 512)) return DMA_ERR_UNSUPPORTED_;
        return uni ? launch(cache_attn_kernel<D, E5M2, MT, 8, true, true>, dim3((unsigned)items), dim3(512), stream, a)
                   : launch(cache_attn_kernel<D, E5M2, MT, 8, true, false>, dim3((unsigned)items), dim3(512), stream, a);
    }
    const int64_t join_y = join_groups(ROWS, a.G, a.s.N);
    if (!few_fit(items, join_y * 1024)) return DMA_ERR_UNSUPPORTED_;
    // the units of the line are counted in 31 bits (at most 2^22 items: some shift suffices)
    while (items * ((a.capacity / STEP >> a.unit_shift) + 2) > 0x7fffffff) ++a.unit_shift;
    const int waves = waves_of(MT, items);
    const int64_t grid = grid_of(waves);
    a.pieces = (float*)workspace;
    a.split = (int2*)(a.pieces + 2 * grid * ROWS * (D + 2));
    const dim3 g((unsigned)grid), block(64 * waves);
    auto go = [&](auto W) {
        return uni ? launch(cache_attn_kernel<D, E5M2, MT, W, false, true>, g, block, stream, a) : launch(cache_attn_kernel<D, E5M2, MT, W, false, false>, g, block, stream, a);
    };
    const int rc = waves == 8 ? go(IC<8>{}) : go(IC<4>{});
    if (rc != DMA_OK_) return rc;
    return launch(cache_attn_join_kernel<D, ROWS>, dim3((unsigned)items, (unsigned)join_y), dim3(1024), stream, a);
}

int launch_cache_attn(const CacheView& c, const Rows& q, const Rows& out, const Spans& s, int Hq, int window, int sinks,
                      void* workspace, hipStream_t stream)
{
    CacheAttnArgs a = {};
    a.c = c;
    a.q = q;
    a.out = out;
    a.s = s;
    a.G = Hq / c.Hkv;
    a.inv_g = (65536u + a.G - 1) / a.G;
    a.window = window;
    a.sinks = window ? sinks : 0;
    a.capacity = c.num_pages ? c.max_pages << c.page_shift : 0;
    a.scale = (float)(1.4426950408889634074 / sqrt((double)c.D));
    if (many_rows(s.B, c.Hkv, a.G, s.N)) return launch_cache_prompt(a, reach_of(c, 128, a.G, window, a.sinks), workspace, stream);
    const int mt = mt_of(a.G, s.N);
    auto pick = [&](auto D, auto F) { return mt == 1 ? launch_few<D, F != 0, 1>(a, workspace, stream) : launch_few<D, F != 0, 2>(a, workspace, stream); };
    if (c.D == 128) return c.e5m2 ? pick(IC<128>{}, IC<1>{}) : pick(IC<128>{}, IC<0>{});
    return c.e5m2 ? pick(IC<64>{}, IC<1>{}) : pick(IC<64>{}, IC<0>{});
}

}  // namespace dma
