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
#include "dma_cache_few.hpp"
#include <algorithm>
#include <atomic>
#include <math.h>

namespace dma {

template <int D, bool E5M2, int MT, int W, bool BY_ITEM, bool UNI>
__global__ void __launch_bounds__(64 * W, 2)
cache_attn_kernel(CacheAttnArgs a)
{
    using Lds = FewLds<D, MT, W>;
    __shared__ __attribute__((aligned(16))) typename Lds::O o;
    __shared__ typename Lds::Ml ml;
    __shared__ __attribute__((aligned(16))) typename Lds::Q q;
    few_rows<D, E5M2, MT, W, BY_ITEM, UNI>(a, Lds{o, ml, q}, OwnAll{}, [](int, unsigned& block, unsigned& blocks) {
        block = blockIdx.x;
        blocks = gridDim.x;
        return true;
    });
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
