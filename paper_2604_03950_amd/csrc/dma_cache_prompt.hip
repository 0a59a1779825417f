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
#include "dma_cache_many.hpp"
#include <algorithm>
#include <math.h>

namespace dma {

template <int D, bool E5M2, int NW, bool UNI>
__global__ void __launch_bounds__(64 * NW, 2)
cache_prompt_kernel(CacheAttnArgs a)
{
    constexpr int ROWS = 32 * NW;
    __shared__ __attribute__((aligned(16))) typename ManyLds<D>::K k_lds;
    __shared__ __attribute__((aligned(16))) typename ManyLds<D>::V v_lds;
    __shared__ int odd[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const CacheView& c = a.c;

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
    const int64_t at = (int64_t)sq.start + tok;
    const int64_t wfirst = (int64_t)sq.start + min(r0, tile * ROWS + rows - 1) / a.G, wlast = (int64_t)sq.start + min(r0 + 31, tile * ROWS + rows - 1) / a.G;
    const int64_t first = (int64_t)sq.start + tile * ROWS / a.G, last = (int64_t)sq.start + (tile * ROWS + rows - 1) / a.G;
    auto behind = [&](int64_t p) { return a.window ? cut_position(p - a.window + 1) : 0; };
    const ManyRows view = {behind(at), cut_position(at), behind(wlast), cut_position(wfirst), behind(wfirst), cut_position(wlast),
                           behind(last), cut_position(first), behind(first), cut_position(last), my_rows};
    v16f o[D / 32];
    float m, l;
    many_steps<D, E5M2, NW, UNI>(a, ManyLds<D>{k_lds, v_lds, odd}, b, h, range, begin, end, view, qf, o, m, l);

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
