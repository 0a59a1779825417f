// Attention over the paged 8-bit cache for many query rows per kv head (pieces of prompts): bound by matrix and vector work.
//
// A workgroup of NW waves takes 32 * NW rows (query tokens times the query heads of a kv head, token by token); every wave has 32 of
// them, and all walk the same steps of 64 positions.  The codes of a step are decoded to bf16 once per workgroup, into LDS (exact: the
// page's scale is applied), one step ahead of their use; one barrier per step.  As in the kernel for few rows, S^T = K Q^T takes its key
// rows in an order that leaves every probability in the lane that needs it for O^T = V^T P^T, and the softmax's maximum is raised only
// where the sum of a lane's 32 probabilities exceeds 1024.  Probabilities are rounded to bf16 as there, for the same reason; here a second term of
// theirs would lengthen by half the products that bound the kernel.
//
// Measured, 32 query and 8 kv heads, D = 128: 2048 tokens behind 14k 530 to 590 us = 0.87 to 0.97 PFLOP/s, 4096 behind 28k 0.98 (a bf16 matrix product
// of 8192^3 runs at 1.15 here); 512 behind 7.5k 91 us = 0.73; 8192 under a window of 1024 180 to 205 us, 0.63 to 0.72 of the visible pairs' flops.  Two
// workgroups of four waves per CU: while one waits at the barrier the other's products run; matrix and vector time of a SIMD add up otherwise.
#include "dma_cache_device.hpp"
#include <algorithm>
#include <math.h>

namespace dma {

// UNI: pages of 64 positions and more, so that a step lies in one: its address is the same for all threads.
template <int D, bool E5M2, int NW, bool UNI>
__global__ void __launch_bounds__(64 * NW, 2)
cache_prompt_kernel(CacheAttnArgs a)
{
    constexpr int ROWS = 32 * NW, T = 64 * NW;
    constexpr int KCH = 64 * (D / 16) / T, VCH = D * 4 / T;       // chunks of 16 codes per thread and step
    constexpr int KROW = 2 * D, VROW = 128;                       // bytes of a row in LDS: a key, a channel's 64 positions
    static_assert(KCH >= 1 && VCH >= 1, "");
    __shared__ __attribute__((aligned(16))) char kbuf[2][64 * KROW], vbuf[2][D * VROW];
    __shared__ int odd_in[4];        // of step j at j & 3: bits 0 to 3: 16 positions without a page, bit 4: a value that is no number
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const CacheView& c = a.c;
    const int page_mask = (1 << c.page_shift) - 1;

    // the last tiles of a sequence have the most keys: first
    unsigned item = blockIdx.x;
    const int part = item % (unsigned)a.parts;
    item /= (unsigned)a.parts;
    const int h = item % (unsigned)c.Hkv;
    item /= (unsigned)c.Hkv;
    const int b = item % (unsigned)a.s.B, tile = a.row_tiles - 1 - (int)(item / (unsigned)a.s.B);
    const SeqInfo sq = seq_of(a, b);
    const int rows = (int)min((int64_t)sq.n * a.G - (int64_t)tile * ROWS, (int64_t)ROWS);
    if (rows <= 0) return;
    const StepRange range = range_of<ROWS, false>(a, sq, tile);
    // the steps of this piece
    const int parts = parts_of(range.steps, a.parts);
    if (part >= parts) return;
    const int begin = (int)((int64_t)range.steps * part / parts), end = (int)((int64_t)range.steps * (part + 1) / parts);

    // ---- rows of this wave
    const int r0 = tile * ROWS + wave * 32, my_rows = min(rows - wave * 32, 32);      // (none: the wave only helps)
    const int row = min(r0 + col, tile * ROWS + rows - 1), tok = row / a.G;
    v8bf qf[D / 16];
    {
        const char* qp = a.q.data + b * a.q.stride_batch + (h * a.G + row - tok * a.G) * a.q.stride_head + tok * a.q.stride_token;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const v8bf*)(qp + (ks * 16 + half * 8) * 2);
    }
    auto cut = [](int64_t p) { return (int)min(max(p, (int64_t)0), (int64_t)POS_MAX); };
    const int64_t at = (int64_t)sq.start + tok;
    const int vis_hi = cut(at), vis_lo = a.window ? cut(at - a.window + 1) : 0;
    // what all rows of the wave see, and what none of the workgroup does
    const int64_t wfirst = (int64_t)sq.start + min(r0, tile * ROWS + rows - 1) / a.G, wlast = (int64_t)sq.start + min(r0 + 31, tile * ROWS + rows - 1) / a.G;
    const int all_hi = cut(wfirst), all_lo = a.window ? cut(wlast - a.window + 1) : 0;
    const int any_hi = cut((int64_t)sq.start + (tile * ROWS + rows - 1) / a.G);
    const int any_lo = a.window ? cut((int64_t)sq.start + tile * ROWS / a.G - a.window + 1) : 0;
    // ... what all of the workgroup see
    const int wg_hi = cut((int64_t)sq.start + tile * ROWS / a.G), wg_lo = a.window ? cut((int64_t)sq.start + (tile * ROWS + rows - 1) / a.G - a.window + 1) : 0;
    // ... of the wave: steps without any visible position are skipped
    const int some_lo = a.window ? cut(wfirst - a.window + 1) : 0, some_hi = cut(wlast);

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
                *(v8bf*)(kbuf[buf] + key * KROW + ((2 * d16 + e) ^ shift) * 16) = decode8<E5M2>(cd.k[u][2 * e], cd.k[u][2 * e + 1], sc);
        }
        // Where not all rows see all positions: values that no row sees may be anything, and a NaN among the others must not reach the
        // rows that do not see it through a probability of zero.  Zeros instead; NaN is put into the sums of those who see it below.  Nor may
        // the scale that zeros are decoded with be anything, where the page is missing or no row sees any of it: with 255 they become NaN.
        const bool open = pos + STEP - 1 <= wg_hi && (pos >= wg_lo || pos + STEP <= a.sinks);
        int odd = 0;
#pragma unroll
        for (int u = 0; u < VCH; ++u) {
            const int ch = threadIdx.x + u * T, d = channel_of(ch);
            float sc = __int_as_float(cd.vsc[UNI ? 0 : u] << 23);
            const bool there = cd.there[UNI ? 0 : u];
            if (!there) odd |= 1 << (ch & 3);
            if (!open || !there) {
                auto below = [&](int q) { return (1u << min(max(q - pos - (ch & 3) * 16, 0), 16)) - 1u; };
                const unsigned seen = there ? below(any_hi + 1) & (~below(any_lo) | below(a.sinks)) : 0u;
                if (!seen) sc = 1.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    cd.v[u][w] &= bytes_of(seen >> (4 * w));
                    const unsigned bad = no_number<E5M2>((unsigned)cd.v[u][w]);
                    if (bad) odd |= 16;
                    cd.v[u][w] &= (int)~((bad >> 7) * 0xffu);
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *(v8bf*)(vbuf[buf] + d * VROW + ((2 * (ch & 3) + e) ^ shift_of(d, VROW)) * 16) = decode8<E5M2>(cd.v[u][2 * e], cd.v[u][2 * e + 1], sc);
        }
        if (odd) atomicOr(&odd_in[j & 3], odd);
    };

    v16f o[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    float m = M_NONE, l = 0.f;

    if (threadIdx.x < 4) odd_in[threadIdx.x] = 0;
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
        if (threadIdx.x == 0) odd_in[(j + 2) & 3] = 0;            // last read two steps ago, next written in the next one
        const int odd = odd_in[j & 3];
        const bool none = my_rows <= 0 || pos > some_hi || (pos + STEP <= some_lo && pos >= a.sinks);
        if (!none) {
            // ---- scores
            v16f s[2];
            v8bf kf[2][D / 16];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const char* kp = kbuf[buf] + (kt * 32 + key_of_row) * KROW;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) kf[kt][ks] = *(const v8bf*)(kp + ((2 * ks + half) ^ shift_of(col, KROW)) * 16);
            }
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
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
                for (int r = 0; r < 16; ++r) x[kt][r] = s[kt][r];
            // ---- what is not seen
            const bool plain = pos + STEP - 1 <= all_hi && (pos >= all_lo || pos + STEP <= a.sinks) && (odd & 15) == 0;
            if (!plain) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    unsigned seen = 0;                            // bit 8 e + i: position kt * 32 + 16 e + 8 half + i
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int base = pos + kt * 32 + 16 * e + 8 * half;
                        auto below = [&](int q) { return (1u << min(max(q - base, 0), 8)) - 1u; };
                        const unsigned f = (below(vis_hi + 1) & (~below(vis_lo) | below(a.sinks))) & 0xffu;
                        seen |= ((odd >> (2 * kt + e)) & 1 ? 0u : f) << (8 * e);
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) x[kt][r] = (seen >> r) & 1u ? x[kt][r] : -INFINITY;
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
                    for (int r = 0; r < 16; ++r) top = fmaxf(top, x[kt][r]);
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
                const unsigned long long hit = nan_channels<D, E5M2>(a, b, h, pos, vis_lo, vis_hi, D / 2, [&](int i) { return (i >> 4) * 32 + 8 * (i >> 2 & 3) + 4 * half + (i & 3); });
#pragma unroll
                for (int i = 0; i < D / 2; ++i) o[i >> 4][i & 15] = (hit >> i) & 1 ? NAN : o[i >> 4][i & 15];
            }
            v8bf vf[D / 32][4];
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) vf[dt][ks] = *(const v8bf*)(vbuf[buf] + (dt * 32 + col) * VROW + ((2 * ks + half) ^ shift_of(col, VROW)) * 16);
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

    if (col >= my_rows) return;
    l = cross_half_sum(l);
    if (parts > 1) {
        const unsigned index = ((unsigned)b * c.Hkv + h) * a.row_tiles + tile;
        float* p = a.pieces + ((int64_t)index * a.parts + part) * (ROWS * (D + 2));
        const int rr = wave * 32 + col;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(v4f*)(p + rr * D + dt * 32 + 8 * q + 4 * half) = v4f{o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]};
        if (half == 0) {
            p[ROWS * D + rr] = m;
            p[ROWS * D + ROWS + rr] = l;
        }
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    char* op = a.out.data + b * a.out.stride_batch + (h * a.G + row - tok * a.G) * a.out.stride_head + tok * a.out.stride_token;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *(v2i*)(op + (dt * 32 + 8 * q + 4 * half) * 2) = v2i{pack_bf16(o[dt][4 * q] * inv, o[dt][4 * q + 1] * inv), pack_bf16(o[dt][4 * q + 2] * inv, o[dt][4 * q + 3] * inv)};
}

constexpr int PROMPT_WAVES = 4, PROMPT_ROWS = 32 * PROMPT_WAVES;

// Joins the pieces of items in several: the workgroups of an item (gridDim.y of them) share its rows, a thread has 4 channels of a row at a time.
template <int D>
__global__ void __launch_bounds__(512)
cache_parts_join_kernel(CacheAttnArgs a)
{
    constexpr int CH = D / 4, ROWS = PROMPT_ROWS, U = 8;
    unsigned item = blockIdx.x;
    const int tile = item % (unsigned)a.row_tiles;
    const int h = item / (unsigned)a.row_tiles % (unsigned)a.c.Hkv, b = item / (unsigned)a.row_tiles / (unsigned)a.c.Hkv;
    const SeqInfo sq = seq_of(a, b);
    const int rows = (int)min((int64_t)sq.n * a.G - (int64_t)tile * ROWS, (int64_t)ROWS);
    if (rows <= 0) return;
    const int parts = parts_of(range_of<ROWS, false>(a, sq, tile).steps, a.parts);
    if (parts == 1) return;
    const float* first = a.pieces + (int64_t)item * a.parts * (ROWS * (D + 2));
    for (int at = blockIdx.y * 512 + threadIdx.x; at < rows * CH; at += gridDim.y * 512) {
        const int rr = at / CH, ch = at % CH;
        v4f o = {0.f, 0.f, 0.f, 0.f};
        float m = M_NONE, l = 0.f;
        for (int w = 0; w < parts; w += U) {
            float m2[U], l2[U];
            v4f x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                m2[u] = M_NONE;
                l2[u] = 0.f;
                x[u] = v4f{0.f, 0.f, 0.f, 0.f};
                if (w + u < parts) {                                      // the same for all threads
                    const float* p = first + (int64_t)(w + u) * (ROWS * (D + 2));
                    m2[u] = p[ROWS * D + rr];
                    l2[u] = p[ROWS * D + ROWS + rr];
                    x[u] = *(const v4f*)(p + rr * D + ch * 4);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (w + u >= parts) break;
                const float up = fmaxf(m, m2[u]);
                const float f1 = __builtin_amdgcn_exp2f((m - up) * a.scale), f2 = __builtin_amdgcn_exp2f((m2[u] - up) * a.scale);
                m = up;
                l = l * f1 + l2[u] * f2;
                o = o * f1 + x[u] * f2;
            }
        }
        const int r = tile * ROWS + rr, i = r / a.G;
        char* op = a.out.data + b * a.out.stride_batch + (h * a.G + r - i * a.G) * a.out.stride_head + i * a.out.stride_token;
        const v4f x = o * (l == 0.f ? 0.f : 1.f / l);
        *(v2i*)(op + ch * 8) = v2i{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    }
}

static int64_t prompt_items(int B, int Hkv, int G, int N) { return (int64_t)B * Hkv * (((int64_t)N * G + PROMPT_ROWS - 1) / PROMPT_ROWS); }

// Pieces per item: as many workgroups as the chip holds (two per CU), where there are fewer items, of at least two of the steps that an item
// can reach.  (16 items of 128 steps: 33.0 us in the other kernel's shares, 28.6 in 32 pieces; 128 items of 125 steps 188 us whole, 103 in 4.)
static int prompt_parts(int B, int Hkv, int G, int N, int64_t reach)
{
    const int64_t most = std::min<int64_t>(32, reach / STEP / 2);
    return (int)std::max<int64_t>(1, std::min(most, 2 * cache_cus() / prompt_items(B, Hkv, G, N)));
}

size_t cache_prompt_workspace(int B, int Hkv, int G, int N, int D, int64_t reach)
{
    const int parts = prompt_parts(B, Hkv, G, N, reach);
    return parts > 1 ? (size_t)(prompt_items(B, Hkv, G, N) * parts * PROMPT_ROWS * (D + 2) * 4) : 0;
}

int launch_cache_prompt(CacheAttnArgs a, int64_t reach, void* workspace, hipStream_t stream)
{
    constexpr int NW = PROMPT_WAVES;
    const int64_t items = prompt_items(a.s.B, a.c.Hkv, a.G, a.s.N);
    a.row_tiles = (int)(items / a.s.B / a.c.Hkv);
    a.parts = prompt_parts(a.s.B, a.c.Hkv, a.G, a.s.N, reach);
    a.pieces = (float*)workspace;
    if (items * a.parts * 64 * NW > 0xffffffffLL) return DMA_ERR_UNSUPPORTED_;
    const dim3 grid((unsigned)(items * a.parts)), block(64 * NW);
    auto go = [&](auto D, auto E5M2) {
        int rc = a.c.page_shift >= 6 ? launch(cache_prompt_kernel<D, E5M2 != 0, NW, true>, grid, block, stream, a)
                                     : launch(cache_prompt_kernel<D, E5M2 != 0, NW, false>, grid, block, stream, a);
        if (rc == DMA_OK_ && a.parts > 1)
            rc = launch(cache_parts_join_kernel<D>, dim3((unsigned)items, (unsigned)std::min(a.parts, PROMPT_ROWS * D / 4 / 512)), dim3(512), stream, a);
        return rc;
    };
    if (a.c.D == 128) return a.c.e5m2 ? go(IC<128>{}, IC<1>{}) : go(IC<128>{}, IC<0>{});
    return a.c.e5m2 ? go(IC<64>{}, IC<1>{}) : go(IC<64>{}, IC<0>{});
}

}  // namespace dma
