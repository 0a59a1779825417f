// What the kernels of the attention over the paged 8-bit cache share.
#pragma once

#include "dma_device.hpp"
#include "dma_internal.hpp"

namespace dma {

constexpr int STEP = 64;                     // positions of a step
constexpr int POS_MAX = 1 << 30;             // above every position that a table holds
constexpr float M_NONE = -3.0e38f;           // the maximum of nothing: below every score, and finite

struct CacheAttnArgs {
    CacheView c;
    Rows q, out;
    Spans s;
    int G;                   // query heads per kv head
    unsigned inv_g;          // ceil(2^16 / G)
    int unit_shift;          // few rows: the line of all items' steps is cut in units of 1 << unit_shift of them
    int row_tiles;           // of a sequence with N tokens
    int window, sinks;
    int capacity;            // positions that a reader may find
    float scale;             // log2(e) / sqrt(D)
    float* pieces;           // of split items: [ROWS][D] sums, then [ROWS] maxima, then [ROWS] weights.  Few rows: 2 per workgroup
    int2* split;             // few rows: per item the first and last workgroup that has a piece (first = last: no pieces)
    int parts;               // many rows: pieces of an item at most, side by side
};

// A word of a table that no kernel running at the same time writes, at an index that is the same for all lanes: by way of the scalar cache, whose loads are counted
// apart from those of the codes.
DMA_DEV int scalar_at(const int* table, int index)
{
    return ((const __attribute__((address_space(4))) int*)(uintptr_t)table)[index];
}

struct SeqInfo {
    int start, n;
};
DMA_DEV SeqInfo seq_of(const CacheAttnArgs& a, int b)
{
    SeqInfo q;
    q.start = a.s.start[b];
    q.n = a.s.n_tokens ? min(max(a.s.n_tokens[b], 0), a.s.N) : a.s.N;
    if (q.start < 0) q.n = 0;
    return q;
}

// Token of a query row, counted from the row tile's first: a multiplication where the rows of a sequence are few (exact below 2^12 rows).
template <bool FEW>
DMA_DEV int token_of(const CacheAttnArgs& a, int row) { return FEW ? (int)((unsigned)row * a.inv_g >> 16) : row / a.G; }

// The steps that a row tile visits: [0, sink_steps) and [first, first + steps - sink_steps).  ONE: a sequence has one tile.
struct StepRange {
    int sink_steps, first, steps;
    DMA_DEV int position(int j) const { return (j < sink_steps ? j : first + j - sink_steps) * STEP; }
};
template <int ROWS, bool ONE>
DMA_DEV StepRange range_of(const CacheAttnArgs& a, const SeqInfo& q, int tile)
{
    const int64_t from = (int64_t)q.start + (ONE ? 0 : tile * ROWS / a.G), to = (int64_t)q.start + (ONE ? q.n - 1 : min(q.n - 1, (tile * ROWS + ROWS - 1) / a.G));
    const int hi = (int)min(to + 1, (int64_t)a.capacity);
    const int lo = a.window ? (int)min(max(from - a.window + 1, (int64_t)0), (int64_t)hi) : 0;
    StepRange r;
    r.first = lo / STEP;
    r.sink_steps = (min(a.sinks, hi) + STEP - 1) / STEP;
    if (r.sink_steps >= r.first) r.sink_steps = r.first = 0;
    r.steps = r.sink_steps + (hi + STEP - 1) / STEP - r.first;
    return r;
}

// Two codes (the lower or upper half of a dword) -> two bf16, times the scale: exact.
template <bool E5M2, bool HI>
DMA_DEV int decode2(int w, float sc)
{
    if constexpr (E5M2) return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((unsigned)w, sc, HI));
    else return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w, sc, HI));
}
// Eight codes -> eight bf16, an operand of the matrix instruction.
template <bool E5M2>
DMA_DEV v8bf decode8(int lo, int hi, float sc)
{
    v4i r;
    r[0] = decode2<E5M2, false>(lo, sc);
    r[1] = decode2<E5M2, true>(lo, sc);
    r[2] = decode2<E5M2, false>(hi, sc);
    r[3] = decode2<E5M2, true>(hi, sc);
    return __builtin_bit_cast(v8bf, r);
}
DMA_DEV float cross_group_max(float x) { return cross_half_max(row_pair_max(x)); }
DMA_DEV float cross_group_sum(float x)
{
    const v2u r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return cross_half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
DMA_DEV int pack_bf16(float a, float b)
{
    v2bf r;
    r[0] = (__bf16)a;
    r[1] = (__bf16)b;
    return __builtin_bit_cast(int, r);
}

// Codes that are no number under their page's scale: bit 7 of each byte.  NaN and infinity in the format, from its code `least` on; under a scale above
// those that a write leaves, also what reaches 2^128, which bf16 does not hold: an exponent field of 128 + bias - (scale - 127); with 255, the
// byte of NaN, every code.  All are put into the sums as NaN where a step is masked; in the others an infinity goes through the products as one.
// limit: what brings the codes from there on to bit 7 when it is added to each.
template <bool E5M2>
DMA_DEV unsigned no_number_limit(int scale)
{
    constexpr int least = E5M2 ? 0x7c : 0x7f, bias = E5M2 ? 15 : 7, mantissa = E5M2 ? 2 : 3;
    return (unsigned)(128 - (scale == 255 ? 0 : min(least, (255 + bias - scale) << mantissa))) * 0x01010101u;
}
DMA_DEV unsigned no_number(unsigned w, unsigned limit) { return ((w & 0x7f7f7f7fu) + limit) & 0x80808080u; }

// Bits 0 to 3 -> the four bytes of a dword.
DMA_DEV int bytes_of(unsigned bits) { return (int)((((bits & 15u) * 0x00204081u) & 0x01010101u) * 0xffu); }

// Which of a lane's channels have a value that is no number at a position that its row sees, among the 64 from pos: bit i for
// channel(i).  Read from the cache, a channel after the other: a NaN must reach the rows that see it and, multiplied by a
// probability of zero, no other, so it is taken out of the matrix product and put into the sums by hand.  Rare, and not fast.
template <int D, bool E5M2, typename F>
DMA_DEV unsigned long long nan_channels(const CacheAttnArgs& a, int b, int h, int pos, int vis_lo, int vis_hi, int n, F&& channel)
{
    unsigned long long hit = 0;
#pragma unroll 1
    for (int g = 0; g < 4; ++g) {
        const int p = pos + 16 * g, pi = p >> a.c.page_shift;
        const int page = pi < a.c.max_pages ? a.c.page_table[(int64_t)b * a.c.max_pages + pi] : -1;
        if ((unsigned)page >= a.c.page_limit) continue;
        auto below = [&](int at) { return (1u << min(max(at - p, 0), 16)) - 1u; };
        const unsigned seen = below(vis_hi + 1) & (~below(vis_lo) | below(a.sinks));
        const int64_t slab = (int64_t)page * a.c.Hkv + h;
        const uint8_t* base = a.c.v_codes + (((slab * D) << a.c.page_shift) + (p & ((1 << a.c.page_shift) - 1)));
        const unsigned limit = no_number_limit<E5M2>(a.c.v_scales[slab]);
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const v4i w = *(const v4i*)(base + (channel(i) << a.c.page_shift));
            unsigned bad = 0;
            for (int k = 0; k < 4; ++k) bad |= no_number((unsigned)w[k], limit) & (unsigned)bytes_of(seen >> (4 * k));
            if (bad) hit |= 1ull << i;
        }
    }
    return hit;
}

// Many query rows (dma_cache_prompt.hip): the steps of an item of 128 rows in `parts` pieces at most, of two steps at least.  reach: the most
// positions that an item can visit.
DMA_DEV int parts_of(int steps, int parts) { return max(min(parts, steps / 2), 1); }
size_t cache_prompt_workspace(int B, int Hkv, int G, int N, int D, int64_t reach);
int launch_cache_prompt(CacheAttnArgs a, int64_t reach, void* workspace, hipStream_t stream);

// Compute units of the current device (256 where it cannot be asked).
int cache_cus();

}  // namespace dma
