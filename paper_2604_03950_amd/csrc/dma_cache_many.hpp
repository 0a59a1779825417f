// The steps of 128 query rows over the paged 8-bit cache, for the kernels that have many rows per kv head: of one sequence's tokens
// (dma_cache_prompt.hip), or of all sequences that share a prefix (dma_cache_shared.hip).  What it does and measures is said at the first.
#pragma once

#include "dma_cache_device.hpp"
#include <math.h>

namespace dma {

template <int D>
struct ManyLds {
    using K = char[2][64 * 2 * D];
    using V = char[2][D * 128];
    K& k;
    V& v;
    int (&odd)[4];           // of step j at j & 3: bits 0 to 3: 16 positions without a page, bit 4: a value that is no number
    int* some = nullptr;     // [4][waves], of step j at j & 3: bits 0 to 3: 16 positions of which a row of the wave sees one
};

// What is visible: positions [vis_lo, vis_hi] and those below the sinks to the row of this lane's column, ...
struct ManyRows {
    int vis_lo, vis_hi;
    int all_lo, all_hi;      // to all rows of the wave
    int some_lo, some_hi;    // to any of them: steps without a visible position are skipped
    int wg_lo, wg_hi;        // to all rows of the workgroup
    int any_lo, any_hi;      // to any of them
    int my_rows;             // of the wave (none: it only helps)
};
DMA_DEV int cut_position(int64_t p) { return (int)min(max(p, (int64_t)0), (int64_t)POS_MAX); }

// Steps [begin, end) of the range, by the pages of sequence b: into sums o, maximum m and weight l of a lane's part of its row (the other half of
// the wave has the other).  GAPS: under a window, positions between those that rows see may be seen by none (rows of several sequences).  UNI: pages of 64 positions and more, so that a step lies in one: its address is the same for all threads.
template <int D, bool E5M2, int NW, bool UNI, bool GAPS = false>
DMA_DEV void many_steps(const CacheAttnArgs& a, const ManyLds<D>& lds, int b, int h, const StepRange& range, int begin, int end, const ManyRows& r,
                        v8bf (&qf)[D / 16], v16f (&o)[D / 32], float& m, float& l)
{
    constexpr int T = 64 * NW;
    constexpr int KCH = 64 * (D / 16) / T, VCH = D * 4 / T;       // chunks of 16 codes per thread and step
    constexpr int KROW = 2 * D, VROW = 128;                       // bytes of a row in LDS: a key, a channel's 64 positions
    static_assert(KCH >= 1 && VCH >= 1, "");
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const CacheView& c = a.c;
    const int page_mask = (1 << c.page_shift) - 1;

    // ---- codes of a step, from memory to registers and from there to LDS
    const int* table = c.page_table + (int64_t)b * c.max_pages;
    struct Pages {
        int k[UNI ? 1 : KCH], v[UNI ? 1 : VCH];
    };
    struct Codes {
        v4i k[KCH], v[VCH];
        uint8_t ksc[UNI ? 1 : KCH], vsc[UNI ? 1 : VCH];
        bool there[UNI ? 1 : VCH];
    };
    auto page_at = [&](int p) -> int {
        const int pi = p >> c.page_shift, at = min(pi, c.max_pages - 1);
        const int page = UNI ? scalar_at(table, at) : table[at];
        return pi < c.max_pages ? page : -1;
    };
    // Which 16 codes a thread has: 8 lanes write to LDS in one turn, and would find half of its banks with 8 chunks of a key (every second
    // one of a row) or 4 of two channels (whose rows are shifted alike): 4 of a key and 4 of the next, 4 of a channel and 4 of the next but one
    // (4096 tokens behind 28k 2062 us, 2086 without).
    auto next_but_one = [](int row) { return (row & ~3) | (row & 1) << 1 | (row >> 1 & 1); };
    auto key_of = [&](int ch) { return D == 128 ? (ch >> 2 & 1) | ch >> 4 << 1 : next_but_one(ch / 4); };
    auto part_of = [](int ch) { return D == 128 ? (ch & 3) | (ch >> 1 & 4) : ch & 3; };
    auto channel_of = [&](int ch) { return next_but_one(ch / 4); };
    auto load_pages = [&](int j, Pages& pg) {                     // one step before load(), two before stage()
        const int pos = range.position(j);
        if constexpr (UNI) pg.k[0] = page_at(pos);
        else {
#pragma unroll
            for (int u = 0; u < KCH; ++u) pg.k[u] = page_at(pos + key_of(threadIdx.x + u * T));
#pragma unroll
            for (int u = 0; u < VCH; ++u) pg.v[u] = page_at(pos + (threadIdx.x & 3) * 16);
        }
    };
    const unsigned kofs = key_of(threadIdx.x) * D + part_of(threadIdx.x) * 16, vofs = (channel_of(threadIdx.x) << c.page_shift) + (threadIdx.x & 3) * 16;
    auto load = [&](int j, const Pages& pg, Codes& cd) {
        const int pos = range.position(j);
        if constexpr (UNI) {
            cd.there[0] = (unsigned)pg.k[0] < c.page_limit;
            const int64_t slab = (int64_t)(cd.there[0] ? pg.k[0] : 0) * c.Hkv + h;
            const uint8_t* kb = c.k_codes + ((slab << c.page_shift) + (pos & page_mask)) * D;
            const uint8_t* vb = c.v_codes + ((slab * D) << c.page_shift) + (pos & page_mask);
#pragma unroll
            for (int u = 0; u < KCH; ++u) cd.k[u] = *(const v4i*)(kb + u * T * 16 + kofs);
#pragma unroll
            for (int u = 0; u < VCH; ++u) cd.v[u] = *(const v4i*)(vb + ((u * T / 4) << c.page_shift) + vofs);
            cd.ksc[0] = c.k_scales[slab];
            cd.vsc[0] = c.v_scales[slab];
        } else {
#pragma unroll
            for (int u = 0; u < KCH; ++u) {
                const int ch = threadIdx.x + u * T, p = pos + key_of(ch);
                const int64_t slab = (int64_t)((unsigned)pg.k[u] < c.page_limit ? pg.k[u] : 0) * c.Hkv + h;
                cd.k[u] = *(const v4i*)(c.k_codes + (((slab << c.page_shift) + (p & page_mask)) * D + part_of(ch) * 16));
                cd.ksc[u] = c.k_scales[slab];
            }
#pragma unroll
            for (int u = 0; u < VCH; ++u) {
                const int ch = threadIdx.x + u * T, p = pos + (ch & 3) * 16;
                cd.there[u] = (unsigned)pg.v[u] < c.page_limit;
                const int64_t slab = (int64_t)(cd.there[u] ? pg.v[u] : 0) * c.Hkv + h;
                cd.v[u] = *(const v4i*)(c.v_codes + (((slab * D + channel_of(ch)) << c.page_shift) + (p & page_mask)));
                cd.vsc[u] = c.v_scales[slab];
            }
        }
    };
    // Rows of LDS are shifted in chunks of 16 bytes so that the 16 lanes of a read's turn find different banks (256 bytes of them: one
    // row, or two of 128 bytes): keys by the number of the lane that reads them, channels by theirs.
    auto shift_of = [](int lane_row, int row_bytes) { return row_bytes == 256 ? lane_row & 15 : lane_row >> 1 & 7; };
    auto stage = [&](int j, int buf, Codes& cd) {
        const int pos = range.position(j);
#pragma unroll
        for (int u = 0; u < KCH; ++u) {
            const int ch = threadIdx.x + u * T, key = key_of(ch), d16 = part_of(ch);
            const int shift = shift_of((key & 3) | (key >> 1 & 4) | (key << 1 & 8), KROW);
            const float sc = __int_as_float(cd.ksc[UNI ? 0 : u] << 23);
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *(v8bf*)(lds.k[buf] + key * KROW + ((2 * d16 + e) ^ shift) * 16) = decode8<E5M2>(cd.k[u][2 * e], cd.k[u][2 * e + 1], sc);
        }
        // Where not all rows see all positions: values that no row sees may be anything, and a NaN among the others must not reach the
        // rows that do not see it through a probability of zero.  Zeros instead; NaN is put into the sums of those who see it below.  Nor may
        // the scale that zeros are decoded with be anything, where the page is missing or no row sees any of it: with 255 they become NaN.
        const bool open = pos + STEP - 1 <= r.wg_hi && (pos >= r.wg_lo || pos + STEP <= a.sinks);
        int odd = 0;
#pragma unroll
        for (int u = 0; u < VCH; ++u) {
            const int ch = threadIdx.x + u * T, d = channel_of(ch);
            int scale = cd.vsc[UNI ? 0 : u];
            const bool there = cd.there[UNI ? 0 : u];
            if (!there) odd |= 1 << (ch & 3);
            if (!open || !there) {
                auto below = [&](int q) { return (1u << min(max(q - pos - (ch & 3) * 16, 0), 16)) - 1u; };
                unsigned seen = there ? below(r.any_hi + 1) & (~below(r.any_lo) | below(a.sinks)) : 0u;
                if constexpr (GAPS) {
                    int some = 0;
#pragma unroll
                    for (int w = 0; w < NW; ++w) some |= lds.some[(j & 3) * NW + w];
                    if (a.window && !((some >> (ch & 3)) & 1)) seen = 0;
                }
                if (!seen) scale = 127;
                const unsigned limit = no_number_limit<E5M2>(scale);
                if (scale == 255) scale = 127;                     // (no code stays)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    cd.v[u][w] &= bytes_of(seen >> (4 * w));
                    const unsigned bad = no_number((unsigned)cd.v[u][w], limit);
                    if (bad) odd |= 16;
                    cd.v[u][w] &= (int)~((bad >> 7) * 0xffu);
                }
            }
            const float sc = __int_as_float(scale << 23);
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *(v8bf*)(lds.v[buf] + d * VROW + ((2 * (ch & 3) + e) ^ shift_of(d, VROW)) * 16) = decode8<E5M2>(cd.v[u][2 * e], cd.v[u][2 * e + 1], sc);
        }
        if (odd) atomicOr(&lds.odd[j & 3], odd);
    };

    // (a page of which no row sees anything may have any scale; where one row sees some of 16 positions, the others among them are numbers, or
    // are found not to be)
    auto look = [&](int j) {
        if constexpr (GAPS) {
            if (!a.window) return;
            const int pos = range.position(j);
            int some = 0;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int p = pos + 16 * g;
                if (__any(p <= r.vis_hi && (p + 15 >= r.vis_lo || p < a.sinks))) some |= 1 << g;
            }
            if (lane == 0) lds.some[(j & 3) * NW + (int)(threadIdx.x >> 6)] = some;
        }
    };

#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    m = M_NONE;
    l = 0.f;

    if (threadIdx.x < 4) lds.odd[threadIdx.x] = 0;
    Pages pages;
    Codes codes;
    if (begin < end) {
        // the first two steps' codes are on their way together
        Pages pages1;
        Codes codes0;
        load_pages(begin, pages);
        load_pages(min(begin + 1, end - 1), pages1);
        load(begin, pages, codes0);
        load(min(begin + 1, end - 1), pages1, codes);
        load_pages(min(begin + 2, end - 1), pages);
        look(begin);
        look(begin + 1);
        __syncthreads();
        stage(begin, begin & 1, codes0);
    }
    __syncthreads();
    // S rows of lane half `half`: register 4 q + i is row 8 q + 4 half + i of the 32, and holds position 16 (q / 2) + 8 half + 4 (q & 1) + i
    const int key_of_row = 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
    // the queries have arrived before the loop: no wait for them inside it, which would be one for the codes requested meanwhile
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        v4i w = __builtin_bit_cast(v4i, qf[ks]);
        asm volatile("" : "+v"(w));
        qf[ks] = __builtin_bit_cast(v8bf, w);
    }
    for (int j = begin; j < end; ++j) {
        const int buf = j & 1, pos = range.position(j);
        if (j + 1 < end) {
            stage(j + 1, buf ^ 1, codes);
            if (j + 2 < end) load(j + 2, pages, codes);
            if (j + 3 < end) load_pages(j + 3, pages);
        }
        look(j + 2);
        if (threadIdx.x == 0) lds.odd[(j + 2) & 3] = 0;            // last read two steps ago, next written in the next one
        const int odd = lds.odd[j & 3];
        const bool none = r.my_rows <= 0 || pos > r.some_hi || (pos + STEP <= r.some_lo && pos >= a.sinks);
        if (!none) {
            // ---- scores
            v16f s[2];
            v8bf kf[2][D / 16];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const char* kp = lds.k[buf] + (kt * 32 + key_of_row) * KROW;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) kf[kt][ks] = *(const v8bf*)(kp + ((2 * ks + half) ^ shift_of(col, KROW)) * 16);
            }
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kt][ks], qf[ks], s[kt], 0, 0, 0);
            }
            // half of the operands ahead, the rest between the products
            __builtin_amdgcn_sched_group_barrier(0x100, D / 16, 0);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, D / 16, 0);
            float x[2][16];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[kt][i] = s[kt][i];
            // ---- what is not seen
            const bool plain = pos + STEP - 1 <= r.all_hi && (pos >= r.all_lo || pos + STEP <= a.sinks) && (odd & 15) == 0;
            if (!plain) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    unsigned seen = 0;                            // bit 8 e + i: position kt * 32 + 16 e + 8 half + i
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int base = pos + kt * 32 + 16 * e + 8 * half;
                        auto below = [&](int q) { return (1u << min(max(q - base, 0), 8)) - 1u; };
                        const unsigned f = (below(r.vis_hi + 1) & (~below(r.vis_lo) | below(a.sinks))) & 0xffu;
                        seen |= ((odd >> (2 * kt + e)) & 1 ? 0u : f) << (8 * e);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[kt][i] = (seen >> i) & 1u ? x[kt][i] : -INFINITY;
                }
            }
            // ---- softmax.  The maximum is looked for only where it was too low: the sum of a lane's 32 probabilities shows it
            // (and is a sum of the rounded ones, as the values' sums are)
            v8bf pf[4];                                           // positions 16 e + 8 half + [0, 8) of the step
            float sum;
            auto probabilities = [&] {
                const float off = m * a.scale;
                const v2bf one = __builtin_bit_cast(v2bf, 0x3f803f80);
                float part[2] = {0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    int pw[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float* y = &x[e >> 1][8 * (e & 1) + 2 * i];
                        pw[i] = pack_bf16(__builtin_amdgcn_exp2f(fmaf(y[0], a.scale, -off)), __builtin_amdgcn_exp2f(fmaf(y[1], a.scale, -off)));
                        part[i & 1] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, pw[i]), one, part[i & 1], false);
                    }
                    pf[e] = __builtin_bit_cast(v8bf, v4i{pw[0], pw[1], pw[2], pw[3]});
                }
                sum = part[0] + part[1];
            };
            probabilities();
            if (__any(sum > 1024.f)) {
                float top = x[0][0];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, x[kt][i]);
                const float up = fmaxf(m, cross_half_max(top)), down = __builtin_amdgcn_exp2f((m - up) * a.scale);
                m = up;
                l *= down;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) o[dt] *= down;
                probabilities();
            }
            l += sum;
            // ---- values
            if (odd & 16) {
                const unsigned long long hit = nan_channels<D, E5M2>(a, b, h, pos, r.vis_lo, r.vis_hi, D / 2, [&](int i) { return (i >> 4) * 32 + 8 * (i >> 2 & 3) + 4 * half + (i & 3); });
#pragma unroll
                for (int i = 0; i < D / 2; ++i) o[i >> 4][i & 15] = (hit >> i) & 1 ? NAN : o[i >> 4][i & 15];
            }
            v8bf vf[D / 32][4];
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) vf[dt][ks] = *(const v8bf*)(lds.v[buf] + (dt * 32 + col) * VROW + ((2 * ks + half) ^ shift_of(col, VROW)) * 16);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[dt][ks], pf[ks], o[dt], 0, 0, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 6, 1);
#pragma unroll
            for (int i = 0; i < D / 8 - 6; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 6, 1);
        }
        __syncthreads();
    }
}

}  // namespace dma
