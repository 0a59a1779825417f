// Attention over the paged 8-bit cache for sequences that share a prefix: the plainest form.  A wave has one query row and visits the positions
// that it can see, 64 at a time; for the scores a lane has a position, for the sums it has channels.  Every row reads its own table.
#include "dma_cache_device.hpp"
#include <math.h>

namespace dma {

template <bool E5M2>
DMA_DEV v2f decode2_f32(unsigned w, float sc, bool hi)
{
    if constexpr (E5M2) return hi ? __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(w, sc, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(w, sc, false);
    else return hi ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, sc, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, sc, false);
}

template <int D, bool E5M2>
__global__ void __launch_bounds__(64)
cache_row_kernel(CacheAttnArgs a)
{
    __shared__ __attribute__((aligned(16))) float qs[D], ps[STEP];
    const CacheView& c = a.c;
    const int lane = threadIdx.x;
    unsigned item = blockIdx.x;
    const int i = item % (unsigned)a.s.N;
    item /= (unsigned)a.s.N;
    const int hq = item % (unsigned)(c.Hkv * a.G), b = item / (unsigned)(c.Hkv * a.G), h = hq / a.G;
    const SeqInfo sq = seq_of(a, b);
    if (i >= sq.n) return;
    const __bf16* q = (const __bf16*)(a.q.data + b * a.q.stride_batch + hq * a.q.stride_head + i * a.q.stride_token);
    for (int d = lane; d < D; d += 64) qs[d] = (float)q[d];
    __syncthreads();
    const int64_t p = (int64_t)sq.start + i;
    const int end = (int)min(p + 1, (int64_t)a.capacity), page_mask = (1 << c.page_shift) - 1;
    const int64_t lo = a.window ? p - a.window + 1 : 0;
    float o[D / 64], m = M_NONE, l = 0.f;
    for (int u = 0; u < D / 64; ++u) o[u] = 0.f;
    for (int pos = 0; pos < end; pos += STEP) {
        if (pos + STEP <= lo && pos >= a.sinks) continue;
        // ---- this lane's position
        const int t = pos + lane;
        int page = -1;
        if (t < end && (t >= lo || t < a.sinks)) page = c.page_table[(int64_t)b * c.max_pages + (t >> c.page_shift)];
        const bool seen = (unsigned)page < c.page_limit;
        float x = -INFINITY;
        if (seen) {
            const int64_t slab = (int64_t)page * c.Hkv + h;
            const float sc = __int_as_float(c.k_scales[slab] << 23);
            const v4i* k = (const v4i*)(c.k_codes + ((slab << c.page_shift) + (t & page_mask)) * D);
            x = 0.f;
            for (int d = 0; d < D; d += 16) {
                const v4i w = k[d / 16];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const v2f y0 = decode2_f32<E5M2>((unsigned)w[e], sc, false), y1 = decode2_f32<E5M2>((unsigned)w[e], sc, true);
                    x += y0[0] * qs[d + 4 * e] + y0[1] * qs[d + 4 * e + 1] + y1[0] * qs[d + 4 * e + 2] + y1[1] * qs[d + 4 * e + 3];
                }
            }
            x *= a.scale;
        }
        float top = x;
        for (int s = 32; s; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
        const float up = fmaxf(m, top), down = __builtin_amdgcn_exp2f(m - up);
        const float w = seen ? __builtin_amdgcn_exp2f(x - up) : 0.f;
        float sum = w;
        for (int s = 32; s; s >>= 1) sum += __shfl_xor(sum, s);
        m = up;
        l = l * down + sum;
        for (int u = 0; u < D / 64; ++u) o[u] *= down;
        ps[lane] = w;
        const unsigned long long who = __ballot(seen);
        __syncthreads();
        // ---- this lane's channels
        for (int g = 0; g < 4; ++g) {
            const unsigned mine = (unsigned)(who >> (16 * g)) & 0xffffu;
            if (!mine) continue;
            const int64_t slab = (int64_t)c.page_table[(int64_t)b * c.max_pages + ((pos + 16 * g) >> c.page_shift)] * c.Hkv + h;
            const float sc = __int_as_float(c.v_scales[slab] << 23);
            for (int u = 0; u < D / 64; ++u) {
                const v4i w4 = *(const v4i*)(c.v_codes + ((slab * D + lane + 64 * u) << c.page_shift) + ((pos + 16 * g) & page_mask));
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const v2f y = decode2_f32<E5M2>((unsigned)w4[e / 4], sc, (e & 2) != 0);
                    if (mine >> e & 1) o[u] += ps[16 * g + e] * y[0];
                    if (mine >> e & 2) o[u] += ps[16 * g + e + 1] * y[1];
                }
            }
        }
        __syncthreads();
    }
    __bf16* out = (__bf16*)(a.out.data + b * a.out.stride_batch + hq * a.out.stride_head + i * a.out.stride_token);
    for (int u = 0; u < D / 64; ++u) out[lane + 64 * u] = (__bf16)(l == 0.f ? 0.f : o[u] / l);
}

size_t cache_attn_shared_workspace(const CacheView&, int, int, int, int, int, int) { return 0; }

int launch_cache_attn_shared(const CacheView& c, const Rows& q, const Rows& out, const Spans& s, int Hq, const Groups&, int window, int sinks,
                             void*, hipStream_t stream)
{
    CacheAttnArgs a = {};
    a.c = c;
    a.q = q;
    a.out = out;
    a.s = s;
    a.G = Hq / c.Hkv;
    a.window = window;
    a.sinks = window ? sinks : 0;
    a.capacity = c.num_pages ? c.max_pages << c.page_shift : 0;
    a.scale = (float)(1.4426950408889634074 / sqrt((double)c.D));
    const int64_t rows = (int64_t)s.B * Hq * s.N;
    if (rows * 64 > 0xffffffffLL) return DMA_ERR_UNSUPPORTED_;
    auto go = [&](auto D, auto F) { return launch(cache_row_kernel<D, F != 0>, dim3((unsigned)rows), dim3(64), stream, a); };
    if (c.D == 128) return c.e5m2 ? go(IC<128>{}, IC<1>{}) : go(IC<128>{}, IC<0>{});
    return c.e5m2 ? go(IC<64>{}, IC<1>{}) : go(IC<64>{}, IC<0>{});
}

}  // namespace dma
