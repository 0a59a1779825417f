// Attention over the paged 8-bit cache for many query rows per kv head (pieces of prompts): bound by matrix and vector work.
//
// A workgroup of NW waves takes 32 * NW rows (query tokens times the query heads of a kv head, token by token); every wave has 32 of
// them, and all walk the same steps of 64 positions.  The codes of a step are decoded to bf16 once per workgroup, into LDS (exact: the
// page's scale is applied), one step ahead of their use; one barrier per step.  As in the kernel for few rows, S^T = K Q^T takes its key
// rows in an order that leaves every probability in the lane that needs it for O^T = V^T P^T, and the softmax's maximum is raised only when
// a score exceeds it by 8 units of base 2.
#include "dma_cache_device.hpp"
#include <algorithm>
#include <math.h>

namespace dma {

template <int D, bool E5M2, int NW>
__global__ void __launch_bounds__(64 * NW, 2)
cache_prompt_kernel(CacheAttnArgs a)
{
    constexpr int ROWS = 32 * NW, T = 64 * NW;
    constexpr int KCH = 64 * (D / 16) / T, VCH = D * 4 / T;       // chunks of 16 codes per thread and step
    constexpr int KROW = 2 * D, VROW = 128;                       // bytes of a row in LDS: a key, a channel's 64 positions
    static_assert(KCH >= 1 && VCH >= 1, "");
    __shared__ __attribute__((aligned(16))) char kbuf[2][64 * KROW], vbuf[2][D * VROW];
    __shared__ int odd_in[4];        // of step j at j & 3: bits 0 to 3: 16 positions without a page, bit 4: a value that is no number
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const CacheView& c = a.c;
    const int page_mask = (1 << c.page_shift) - 1;

    // the last tiles of a sequence have the most keys: first
    unsigned item = blockIdx.x;
    const int h = item % (unsigned)c.Hkv;
    item /= (unsigned)c.Hkv;
    const int b = item % (unsigned)a.s.B, tile = a.row_tiles - 1 - (int)(item / (unsigned)a.s.B);
    const SeqInfo sq = seq_of(a, b);
    const int rows = (int)min((int64_t)sq.n * a.G - (int64_t)tile * ROWS, (int64_t)ROWS);
    if (rows <= 0) return;
    const StepRange range = range_of<ROWS>(a, sq, tile);

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
    // ... of the wave: steps without any visible position are skipped
    const int some_lo = a.window ? cut(wfirst - a.window + 1) : 0, some_hi = cut(wlast);

    // ---- codes of a step, from memory to registers and from there to LDS
    const int* table = c.page_table + (int64_t)b * c.max_pages;
    v4i kr[KCH], vr[VCH];
    int kpage[KCH], vpage[VCH], ksc[KCH], vsc[VCH];
    bool vok[VCH];
    auto load_pages = [&](int j) {                                // one step before load(), two before stage()
        const int pos = range.position(j);
        auto page_at = [&](int p) -> int {
            const int pi = p >> c.page_shift;
            return pi < c.max_pages ? table[pi] : -1;
        };
#pragma unroll
        for (int u = 0; u < KCH; ++u) kpage[u] = page_at(pos + (threadIdx.x + u * T) / (D / 16));
#pragma unroll
        for (int u = 0; u < VCH; ++u) vpage[u] = page_at(pos + (threadIdx.x & 3) * 16);
    };
    auto load = [&](int j) {
        const int pos = range.position(j);
#pragma unroll
        for (int u = 0; u < KCH; ++u) {
            const int ch = threadIdx.x + u * T, p = pos + ch / (D / 16);
            const int64_t slab = (int64_t)(kpage[u] < c.num_pages ? max(kpage[u], 0) : 0) * c.Hkv + h;
            kr[u] = *(const v4i*)(c.k_codes + (((slab << c.page_shift) + (p & page_mask)) * D + ch % (D / 16) * 16));
            ksc[u] = c.k_scales[slab];
        }
#pragma unroll
        for (int u = 0; u < VCH; ++u) {
            const int ch = threadIdx.x + u * T, p = pos + (ch & 3) * 16;
            vok[u] = vpage[u] >= 0 && vpage[u] < c.num_pages;
            const int64_t slab = (int64_t)(vok[u] ? vpage[u] : 0) * c.Hkv + h;
            vr[u] = *(const v4i*)(c.v_codes + (((slab * D + ch / 4) << c.page_shift) + (p & page_mask)));
            vsc[u] = c.v_scales[slab];
        }
    };
    auto stage = [&](int j, int buf) {
        const int pos = range.position(j);
#pragma unroll
        for (int u = 0; u < KCH; ++u) {
            const int ch = threadIdx.x + u * T, key = ch / (D / 16), d16 = ch % (D / 16);
            const float sc = __int_as_float(ksc[u] << 23);
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *(v8bf*)(kbuf[buf] + key * KROW + (((2 * d16 + e) ^ (key & (D / 8 - 1))) * 16)) = decode8<E5M2>(kr[u][2 * e], kr[u][2 * e + 1], sc);
        }
        unsigned bad = 0;
        int odd = 0;
#pragma unroll
        for (int u = 0; u < VCH; ++u) {
            const int ch = threadIdx.x + u * T, d = ch / 4, p = pos + (ch & 3) * 16;
            const float sc = __int_as_float(vsc[u] << 23);
            if (!vok[u]) odd |= 1 << (ch & 3);
            // values that no row sees may be anything: zeros instead
            if (!vok[u] || p + 15 > any_hi || (p < any_lo && p + 16 > a.sinks)) {
                auto below = [&](int q) { return (1u << min(max(q - p, 0), 16)) - 1u; };
                const unsigned seen = vok[u] ? below(any_hi + 1) & (~below(any_lo) | below(a.sinks)) : 0u;
#pragma unroll
                for (int w = 0; w < 4; ++w) vr[u][w] &= bytes_of(seen >> (4 * w));
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) bad |= no_number<E5M2>((unsigned)vr[u][w]);
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *(v8bf*)(vbuf[buf] + d * VROW + (((2 * (ch & 3) + e) ^ (d & 7)) * 16)) = decode8<E5M2>(vr[u][2 * e], vr[u][2 * e + 1], sc);
        }
        if (bad) odd |= 16;
        if (odd) atomicOr(&odd_in[j & 3], odd);
    };

    v16f o[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    float m = M_NONE, l = 0.f;

    if (threadIdx.x < 4) odd_in[threadIdx.x] = 0;
    if (range.steps > 0) {
        load_pages(0);
        load(0);
        if (range.steps > 1) load_pages(1);
    }
    __syncthreads();
    if (range.steps > 0) {
        stage(0, 0);
        if (range.steps > 1) load(1);
        if (range.steps > 2) load_pages(2);
    }
    __syncthreads();
    // S rows of lane half `half`: register 4 q + i is row 8 q + 4 half + i of the 32, and holds position 16 (q / 2) + 8 half + 4 (q & 1) + i
    const int key_of_row = 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
    for (int j = 0; j < range.steps; ++j) {
        const int buf = j & 1, pos = range.position(j);
        if (j + 1 < range.steps) {
            stage(j + 1, buf ^ 1);
            if (j + 2 < range.steps) load(j + 2);
            if (j + 3 < range.steps) load_pages(j + 3);
        }
        if (threadIdx.x == 0) odd_in[(j + 2) & 3] = 0;            // last read two steps ago, next written in the next one
        const int odd = odd_in[j & 3];
        const bool none = my_rows <= 0 || pos > some_hi || (pos + STEP <= some_lo && pos >= a.sinks);
        if (!none) {
            // ---- scores
            v16f s[2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
                const int key = kt * 32 + key_of_row;
                const char* kp = kbuf[buf] + key * KROW;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const v8bf k = *(const v8bf*)(kp + (((2 * ks + half) ^ (key & (D / 8 - 1))) * 16));
                    s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[ks], s[kt], 0, 0, 0);
                }
            }
            float x[2][16];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) x[kt][r] = s[kt][r];
            // ---- what is not seen
            const bool plain = pos + STEP - 1 <= all_hi && (pos >= all_lo || pos + STEP <= a.sinks) && (odd & 15) == 0;
            unsigned seen[2] = {0xffffu, 0xffffu};               // bit 8 e + i: position kt * 32 + 16 e + 8 half + i
            if (!plain) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    seen[kt] = 0;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int base = pos + kt * 32 + 16 * e + 8 * half;
                        auto below = [&](int q) { return (1u << min(max(q - base, 0), 8)) - 1u; };
                        const unsigned f = (below(vis_hi + 1) & (~below(vis_lo) | below(a.sinks))) & 0xffu;
                        seen[kt] |= ((odd >> (2 * kt + e)) & 1 ? 0u : f) << (8 * e);
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) x[kt][r] = (seen[kt] >> r) & 1u ? x[kt][r] : -INFINITY;
                }
            }
            // ---- softmax
            float top = x[0][0];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, x[kt][r]);
            if (__any((top - m) * a.scale > 8.f)) {
                const float up = fmaxf(m, cross_half_max(top)), down = __builtin_amdgcn_exp2f((m - up) * a.scale);
                m = up;
                l *= down;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) o[dt] *= down;
            }
            const float off = m * a.scale;
            v8bf pf[4];                                           // positions 16 e + 8 half + [0, 8) of the step
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    int pw[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p0 = __builtin_amdgcn_exp2f(fmaf(x[kt][8 * e + 2 * i], a.scale, -off));
                        const float p1 = __builtin_amdgcn_exp2f(fmaf(x[kt][8 * e + 2 * i + 1], a.scale, -off));
                        l += p0 + p1;
                        pw[i] = pack_bf16(p0, p1);
                    }
                    pf[2 * kt + e] = __builtin_bit_cast(v8bf, v4i{pw[0], pw[1], pw[2], pw[3]});
                }
            // ---- values
            if (!(odd & 16) || plain) {
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) {
                    const int d = dt * 32 + col;
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) {
                        const v8bf v = *(const v8bf*)(vbuf[buf] + d * VROW + (((2 * ks + half) ^ (d & 7)) * 16));
                        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[ks], o[dt], 0, 0, 0);
                    }
                }
            } else {
                // some value is no number: row after row, with what the row does not see taken out
#pragma unroll 1
                for (int r = 0; r < 32; ++r) {
                    const unsigned mine[2] = {(unsigned)__shfl((int)seen[0], (lane & 32) + r), (unsigned)__shfl((int)seen[1], (lane & 32) + r)};
#pragma unroll
                    for (int dt = 0; dt < D / 32; ++dt) {
                        const int d = dt * 32 + col;
                        v16f y;
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] = 0.f;
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks) {
                            const unsigned f = mine[ks >> 1] >> (8 * (ks & 1));
                            v4i v = *(const v4i*)(vbuf[buf] + d * VROW + (((2 * ks + half) ^ (d & 7)) * 16));
#pragma unroll
                            for (int i = 0; i < 4; ++i) v[i] &= (int)(((f >> (2 * i)) & 1u) * 0xffffu | ((f >> (2 * i + 1)) & 1u) * 0xffff0000u);
                            y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, v), pf[ks], y, 0, 0, 0);
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[dt][i] += col == r ? y[i] : 0.f;
                        __builtin_amdgcn_sched_barrier(0);        // one channel tile's operands at a time
                    }
                }
            }
        }
        __syncthreads();
    }

    if (col >= my_rows) return;
    l = cross_half_sum(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    char* op = a.out.data + b * a.out.stride_batch + (h * a.G + row - tok * a.G) * a.out.stride_head + tok * a.out.stride_token;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *(v2i*)(op + (dt * 32 + 8 * q + 4 * half) * 2) = v2i{pack_bf16(o[dt][4 * q] * inv, o[dt][4 * q + 1] * inv), pack_bf16(o[dt][4 * q + 2] * inv, o[dt][4 * q + 3] * inv)};
}

int launch_cache_prompt(CacheAttnArgs a, hipStream_t stream)
{
    constexpr int NW = 4;
    const int64_t tiles = ((int64_t)a.s.N * a.G + 32 * NW - 1) / (32 * NW), items = (int64_t)a.s.B * a.c.Hkv * tiles;
    if (items * 64 * NW > 0xffffffffLL) return DMA_ERR_UNSUPPORTED_;
    a.row_tiles = (int)tiles;
    const dim3 grid((unsigned)items), block(64 * NW);
    if (a.c.D == 128) return a.c.e5m2 ? launch(cache_prompt_kernel<128, true, NW>, grid, block, stream, a) : launch(cache_prompt_kernel<128, false, NW>, grid, block, stream, a);
    return a.c.e5m2 ? launch(cache_prompt_kernel<64, true, NW>, grid, block, stream, a) : launch(cache_prompt_kernel<64, false, NW>, grid, block, stream, a);
}

}  // namespace dma
