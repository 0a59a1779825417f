// Attention over the paged 8-bit cache, the plain way: one wave per query row, 64 keys at a time, a lane per key for the scores
// and a lane per channel (two at D = 128) for the values.  Online softmax in base 2, everything in binary32.
#include "dma_device.hpp"
#include "dma_internal.hpp"
#include <math.h>

namespace dma {

template <bool E5M2>
DMA_DEV float decode1(unsigned byte, float sc)
{
    if constexpr (E5M2) return __builtin_amdgcn_cvt_scalef32_f32_bf8(byte, sc, 0);
    else return __builtin_amdgcn_cvt_scalef32_f32_fp8(byte, sc, 0);
}

template <int D, bool E5M2>
__global__ void __launch_bounds__(64)
cache_attn_row_kernel(CacheView c, Rows q, Rows out, Spans s, int Hq, int window, int sinks, float scale)
{
    const int lane = threadIdx.x;
    unsigned r = blockIdx.x;
    const int h = r % (unsigned)Hq;
    r /= (unsigned)Hq;
    const int i = r % (unsigned)s.N, b = r / (unsigned)s.N;
    const int start = s.start[b], n = s.n_tokens ? min(max(s.n_tokens[b], 0), s.N) : s.N;
    if (start < 0 || i >= n) return;
    const int64_t at = (int64_t)start + i;
    const int end = (int)min(at + 1, (int64_t)c.max_pages << c.page_shift);
    const int64_t from = window ? at - window + 1 : 0;
    const int kvh = h / (Hq / c.Hkv), P = 1 << c.page_shift;
    __shared__ float qs[D], ps[64];
    __shared__ int64_t slabs[64];
    const unsigned short* qp = (const unsigned short*)(q.data + b * q.stride_batch + h * q.stride_head + i * q.stride_token);
    for (int d = lane; d < D; d += 64) qs[d] = __int_as_float((int)qp[d] << 16);
    __syncthreads();
    float m = -INFINITY, l = 0.f, o[D / 64] = {};
    for (int t0 = 0; t0 < end; t0 += 64) {
        const int t = t0 + lane;
        int64_t slab = -1;
        if (t < end && (t >= from || t < sinks)) {
            const int page = c.page_table[(int64_t)b * c.max_pages + (t >> c.page_shift)];
            if (page >= 0 && page < c.num_pages) slab = (int64_t)page * c.Hkv + kvh;
        }
        float x = -INFINITY;
        if (slab >= 0) {
            const uint8_t* row = c.k_codes + ((slab << c.page_shift) + (t & (P - 1))) * D;
            const float sc = __int_as_float((int)c.k_scales[slab] << 23);
            x = 0.f;
            for (int d = 0; d < D; ++d) x = fmaf(qs[d], decode1<E5M2>(row[d], sc), x);
            x *= scale;
        }
        float mx = x;
        for (int w = 32; w; w >>= 1) mx = fmaxf(mx, __shfl_xor(mx, w));
        if (mx == -INFINITY) continue;                            // nothing visible, the same for all lanes
        mx = fmaxf(mx, m);
        const float p = exp2f(x - mx), keep = exp2f(m - mx);
        m = mx;
        float sum = p;
        for (int w = 32; w; w >>= 1) sum += __shfl_xor(sum, w);
        l = l * keep + sum;
        __syncthreads();
        ps[lane] = p;
        slabs[lane] = slab;
        __syncthreads();
        for (int u = 0; u < D / 64; ++u) {
            o[u] *= keep;
            const int d = lane + 64 * u;
            for (int k = 0; k < 64; ++k) {
                const int64_t sl = slabs[k];
                if (sl < 0) continue;
                const float sc = __int_as_float((int)c.v_scales[sl] << 23);
                o[u] = fmaf(ps[k], decode1<E5M2>(c.v_codes[((sl * D + d) << c.page_shift) + ((t0 + k) & (P - 1))], sc), o[u]);
            }
        }
    }
    __bf16* op = (__bf16*)(out.data + b * out.stride_batch + h * out.stride_head + i * out.stride_token);
    for (int u = 0; u < D / 64; ++u) op[lane + 64 * u] = (__bf16)(l > 0.f ? o[u] / l : 0.f);
}

int launch_cache_attn(const CacheView& c, const Rows& q, const Rows& out, const Spans& s, int Hq, int window, int sinks,
                      void*, hipStream_t stream)
{
    using F = void(CacheView, Rows, Rows, Spans, int, int, int, float);
    F* const kernels[2][2] = {{cache_attn_row_kernel<64, false>, cache_attn_row_kernel<64, true>},
                              {cache_attn_row_kernel<128, false>, cache_attn_row_kernel<128, true>}};
    const int64_t blocks = (int64_t)s.B * Hq * s.N;
    if (blocks * 64 > 0xffffffffLL) return DMA_ERR_UNSUPPORTED_;
    return launch(kernels[c.D == 128][c.e5m2], dim3((unsigned)blocks), dim3(64), stream, c, q, out, s, Hq, window, window ? sinks : 0,
                  (float)(1.4426950408889634074 / sqrt((double)c.D)));
}

size_t cache_attn_workspace(int, int, int, int, int) { return 0; }

}  // namespace dma
