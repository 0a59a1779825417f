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

// A word of a table that no kernel writes, at an index that is the same for all lanes: by way of the scalar cache, whose loads are counted
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

// Bytes that are no number (NaN, infinity): bit 7 of each.
template <bool E5M2>
DMA_DEV unsigned no_number(unsigned w) { return ((w & 0x7f7f7f7fu) + (E5M2 ? 0x04040404u : 0x01010101u)) & 0x80808080u; }

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
        const uint8_t* base = a.c.v_codes + (((((int64_t)page * a.c.Hkv + h) * D) << a.c.page_shift) + (p & ((1 << a.c.page_shift) - 1)));
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const v4i w = *(const v4i*)(base + (channel(i) << a.c.page_shift));
            unsigned bad = 0;
            for (int k = 0; k < 4; ++k) bad |= no_number<E5M2>((unsigned)w[k]) & (unsigned)bytes_of(seen >> (4 * k));
            if (bad) hit |= 1ull << i;
        }
    }
    return hit;
}

// Many query rows (dma_cache_prompt.hip): the steps of an item of 128 rows in `parts` pieces at most, of four steps at least.
DMA_DEV int parts_of(int steps, int parts) { return max(min(parts, steps / 4), 1); }
int prompt_parts(int B, int Hkv, int G, int N);
size_t cache_prompt_workspace(int B, int Hkv, int G, int N, int D);
int launch_cache_prompt(CacheAttnArgs a, void* workspace, hipStream_t stream);

// Compute units of the current device (256 where it cannot be asked).
int cache_cus();

// Joins the pieces of split items: a workgroup per item and 4 of its rows; threads over channels (4 each), rows and pieces,
// a thread's loads of several pieces in flight at a time.  Bound by latency: three dependent loads.
// PARTS: the pieces of an item lie side by side, a.parts of them at most; otherwise where a.split says.
template <int D, int ROWS, bool PARTS>
__global__ void __launch_bounds__(1024)
cache_attn_join_kernel(CacheAttnArgs a)
{
    constexpr int CH = D / 4, PG = 1024 / (4 * CH), U = 4;
    unsigned item = blockIdx.x;
    const int tile = item % (unsigned)a.row_tiles;
    const int h = item / (unsigned)a.row_tiles % (unsigned)a.c.Hkv, b = item / (unsigned)a.row_tiles / (unsigned)a.c.Hkv;
    int2 sp = {0, 0};
    if constexpr (!PARTS) sp = a.split[item];                   // anything where the item does not exist
    const SeqInfo sq = seq_of(a, b);
    const int rows = (int)min((int64_t)sq.n * a.G - (int64_t)tile * ROWS, (int64_t)ROWS);
    const int rr = blockIdx.y * 4 + threadIdx.x / CH % 4, ch = threadIdx.x % CH, pg = threadIdx.x / (4 * CH);
    if ((int)blockIdx.y * 4 >= rows) return;
    if constexpr (PARTS) sp.y = parts_of(range_of<ROWS, false>(a, sq, tile).steps, a.parts) - 1;
    if (sp.x == sp.y) return;
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
            const int wu = min(w + u * PG, sp.y);
            const float* p = a.pieces + (PARTS ? (int64_t)item * a.parts + wu : (int64_t)(2 * wu + (wu == sp.x))) * (ROWS * (D + 2));
            m2[u] = p[ROWS * D + r0];
            l2[u] = p[ROWS * D + ROWS + r0];
            x[u] = *(const v4f*)(p + r0 * D + ch * 4);
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

}  // namespace dma
