// The paged 8-bit key / value cache: quantizing as it is written, and reading back.  Both are one pass over their data.
//
// A workgroup takes the keys or the values of one page of one kv head, and holds all of it in registers: a thread has four
// chunks of 8 elements (16 bytes).  For keys, consecutive threads have consecutive chunks; for values a thread's four chunks
// are the same 8 channels of four consecutive positions, so that the codes of a channel are whole dwords (positions lie
// innermost).  A whole page's values go through LDS, where they are turned, and cross memory in one piece.
//
// Bound by memory.  Measured at 32 kv heads x 8192 tokens, D = 128, written (134 MB read, 67 written): 34.4 us = 5.9 TB/s; 8 kv heads x 32768 read
// back: 30.2 us = 6.7 TB/s (a copy of as many bytes 32.5).  One token of 8 kv heads: 4.8 us, one chain of loads.
#include "dma_cache_device.hpp"
#include <algorithm>

namespace dma {

constexpr int CACHE_SCALE_MIN = 17;      // the smallest element of either format times 2^(17 - 127) is a normal bf16 number
DMA_DEV_CONSTEXPR int cache_e_max(bool e5m2) { return e5m2 ? 15 : 8; }
// ... and the largest, 1.75 * 2^e_max, times 2^(scale - 127) is at most 1.75 * 2^127
DMA_DEV_CONSTEXPR int cache_scale_max(bool e5m2) { return 254 - cache_e_max(e5m2); }

// What a workgroup works on.
struct PageItem {
    int b, h, kv;              // sequence, kv head, 0 = keys / 1 = values
    int first;                 // position of the page's first place
    int lo, hi;                // the call's tokens are at places [lo, hi) of the page
    int start;
    int64_t slab;              // index of (page, head)
};
DMA_DEV bool find_item(const CacheView& c, const Spans& s, int pages_per_seq, PageItem& it)
{
    unsigned i = blockIdx.x;
    it.kv = i & 1;
    i >>= 1;
    it.h = i % (unsigned)c.Hkv;
    i /= (unsigned)c.Hkv;
    const int j = i % (unsigned)pages_per_seq;
    it.b = i / (unsigned)pages_per_seq;
    it.start = s.start[it.b];
    const int n = s.n_tokens ? min(max(s.n_tokens[it.b], 0), s.N) : s.N;
    const int P = 1 << c.page_shift, capacity = c.max_pages << c.page_shift;
    if (it.start < 0 || it.start >= capacity || n == 0) return false;
    const int end = (int)min((int64_t)it.start + n, (int64_t)capacity);
    const int pi = (it.start >> c.page_shift) + j;
    it.first = pi << c.page_shift;
    if (it.first >= end) return false;            // (pi < max_pages follows from it)
    const int page = c.page_table[(int64_t)it.b * c.max_pages + pi];
    if ((unsigned)page >= c.page_limit) return false;
    it.lo = max(it.start - it.first, 0);
    it.hi = min(end - it.first, P);
    it.slab = (int64_t)page * c.Hkv + it.h;
    return true;
}

// Dword of the value codes of (channel d, positions 4 quad ..) in LDS: rows of 1 << page_shift bytes.  The rows of a group of 8 channels
// are permuted by the group's number, and the 16-byte chunks of a row by that of 32 channels, so that the threads of a wave (all channel
// groups of 16 or 32 positions) write to different banks.
DMA_DEV int turned(int page_shift, int d, int quad)
{
    return ((d ^ ((d >> 3) & 7)) << (page_shift - 2)) + (quad ^ ((d >> 5) << 2 & ((1 << (page_shift - 2)) - 4)));
}

// Place and channel group of chunk u of this thread.
template <int D>
DMA_DEV void chunk_of(int kv, int page_shift, int u, int& place, int& dch)
{
    if (kv == 0) {
        const int ch = threadIdx.x + u * ((1 << page_shift) / 4 * (D / 8));
        place = ch / (D / 8);
        dch = ch % (D / 8);
    } else {
        place = 4 * (threadIdx.x / (D / 8)) + u;
        dch = threadIdx.x % (D / 8);
    }
}

// Eight bf16 -> eight codes, divided by the power of two in sc, to nearest even.  (By way of binary32: the convert that reads packed bf16
// saves 32 of some 190 vector instructions of a thread and costs time, 64 rows of 128 at a time 42.4 us against 40.0 for 201 MB: the
// kernel is bound by memory.)
template <bool E5M2>
DMA_DEV v2i encode8_cache(const v4i& w, float sc)
{
    float x[8];
    unpack8<false>(w, 1.f, x);
    v2s a = {0, 0}, b = {0, 0};
    if constexpr (E5M2) {
        a = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(a, x[0], x[1], sc, false);
        a = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(a, x[2], x[3], sc, true);
        b = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(b, x[4], x[5], sc, false);
        b = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(b, x[6], x[7], sc, true);
    } else {
        a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[0], x[1], sc, false);
        a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[2], x[3], sc, true);
        b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[4], x[5], sc, false);
        b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[6], x[7], sc, true);
    }
    return v2i{__builtin_bit_cast(int, a), __builtin_bit_cast(int, b)};
}

// Four dwords of four bytes, turned: byte u of r[i] is byte i of w[u].
DMA_DEV void turn4(const unsigned (&w)[4], unsigned (&r)[4])
{
    const unsigned a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
    const unsigned c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    r[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    r[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    r[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    r[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// Four codes rounded once more, to element * 2^-by (by > 0: nothing can overflow).  down: 2^-by.
template <bool E5M2>
DMA_DEV unsigned recode4(unsigned w, float down)
{
    v2s r = {0, 0};
    const float one = cvt_scale_operand(127);
    if constexpr (E5M2) {
        const v2f lo = __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(w, down, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(w, down, true);
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, lo[0], lo[1], one, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, hi[0], hi[1], one, true);
    } else {
        const v2f lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, down, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, down, true);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, lo[0], lo[1], one, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, hi[0], hi[1], one, true);
    }
    return __builtin_bit_cast(unsigned, r);
}

// Largest finite magnitude of eight bf16, as a 15-bit pattern (the rare way: something in them is not finite).
DMA_DEV unsigned amax8_finite(const v4i& w)
{
    unsigned m = 0;
    for (int t = 0; t < 4; ++t) {
        const unsigned a = w[t] & 0x7fff, b = (w[t] >> 16) & 0x7fff;
        if (a < 0x7f80u) m = max(m, a);
        if (b < 0x7f80u) m = max(m, b);
    }
    return m;
}

// Magnitudes above the bf16 pattern `lim` become it, NaN apart.
DMA_DEV v4i clamp8(v4i w, unsigned lim)
{
    for (int t = 0; t < 4; ++t) {
        unsigned r = 0;
        for (int s = 0; s < 32; s += 16) {
            const unsigned x = ((unsigned)w[t] >> s) & 0xffffu, m = x & 0x7fffu;
            r |= ((m > lim && m <= 0x7f80u) ? (x & 0x8000u) | lim : x) << s;
        }
        w[t] = (int)r;
    }
    return w;
}

template <int D, bool E5M2>
__global__ void __launch_bounds__(1024)
kv_write_kernel(CacheView c, Rows k, Rows v, Spans s, int pages_per_seq)
{
    constexpr int EMAX = cache_e_max(E5M2);
    PageItem it;
    if (!find_item(c, s, pages_per_seq, it)) return;            // the same for the whole workgroup
    const Rows& src = it.kv ? v : k;
    uint8_t* codes = (it.kv ? c.v_codes : c.k_codes) + ((it.slab * D) << c.page_shift);
    uint8_t* scale_at = (it.kv ? c.v_scales : c.k_scales) + it.slab;
    const char* row0 = src.data + it.b * src.stride_batch + it.h * src.stride_head;
    const int P = 1 << c.page_shift;
    const bool active = threadIdx.x < (P / 4) * (D / 8);        // all but for pages of 16 at D = 64: half a wave
    v4i w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        int place, dch;
        chunk_of<D>(it.kv, c.page_shift, u, place, dch);
        w[u] = v4i{0, 0, 0, 0};
        if (active && place >= it.lo && place < it.hi)
            w[u] = __builtin_nontemporal_load((const v4i*)(row0 + (int64_t)(it.first + place - it.start) * src.stride_token + dch * 16));
    }
    const unsigned two = pk_max_u16(pk_max_u16(amax8_bf16_packed(w[0]), amax8_bf16_packed(w[1])), pk_max_u16(amax8_bf16_packed(w[2]), amax8_bf16_packed(w[3])));
    unsigned top = max(two & 0xffffu, two >> 16);               // largest finite magnitude, a bf16 pattern
    const bool odd = top > 0x7f60u;                             // something above 1.75 * 2^127
    if (top >= 0x7f80u) top = max(max(amax8_finite(w[0]), amax8_finite(w[1])), max(amax8_finite(w[2]), amax8_finite(w[3])));
    // largest of the workgroup
    __shared__ unsigned wave_top[16];
    top = __float_as_uint(cross_half_max(row_pair_max(group_max<16>(__uint_as_float(top << 16))))) >> 16;
    if ((threadIdx.x & 63) == 0) wave_top[threadIdx.x >> 6] = top;
    int before = it.lo ? *scale_at : 0;                         // every thread reads it before one replaces it
    if (before < CACHE_SCALE_MIN || before > cache_scale_max(E5M2)) before = 0;       // no write left it: the page holds nothing
    __syncthreads();
    for (int i = 0; i < (int)blockDim.x >> 6; ++i) top = max(top, wave_top[i]);
    // the smallest scale that holds it: 1.75 * 2^n and less have significand bits up to 96 of 128
    const int need = min(max((int)((top + 31) >> 7) - EMAX, CACHE_SCALE_MIN), cache_scale_max(E5M2));
    const int scale = max(need, before);
    const bool grown = before && scale > before;
    const float down = __int_as_float((127 - min(scale - before, 100)) << 23);
    if (threadIdx.x == 0) *scale_at = (uint8_t)scale;
    if (!active) return;
    const float sc = cvt_scale_operand(scale);
    v2i q[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (odd) w[u] = clamp8(w[u], min((unsigned)((scale + EMAX) << 7) | 96u, 0x7f60u));
        q[u] = encode8_cache<E5M2>(w[u], sc);
    }
    // whole pages pass the caches by: a prompt is larger than they are (201 MB with its codes kept in them 36.1 us, without 34.2)
    const bool full = it.lo == 0 && it.hi == P;                 // the same for the whole workgroup
    if (it.kv == 0) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            int place, dch;
            chunk_of<D>(0, c.page_shift, u, place, dch);
            v2i* at = (v2i*)(codes + place * D + dch * 8);
            if (full) __builtin_nontemporal_store(q[u], at);
            else if (place >= it.lo && place < it.hi) *at = q[u];
            else if (grown && place < it.lo) {
                v2i old = *at;
                old[0] = (int)recode4<E5M2>((unsigned)old[0], down);
                old[1] = (int)recode4<E5M2>((unsigned)old[1], down);
                *at = old;
            }
        }
    } else {
        int place, dch;
        chunk_of<D>(1, c.page_shift, 0, place, dch);
        uint8_t* col = codes + ((dch * 8) << c.page_shift) + place;
        unsigned w4[8];                                         // of channel i, the four positions
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const unsigned in[4] = {(unsigned)q[0][i >> 2], (unsigned)q[1][i >> 2], (unsigned)q[2][i >> 2], (unsigned)q[3][i >> 2]};
            unsigned r[4];
            turn4(in, r);
            w4[i] = r[0]; w4[i + 1] = r[1]; w4[i + 2] = r[2]; w4[i + 3] = r[3];
        }
        if (full) {
            extern __shared__ __attribute__((aligned(16))) unsigned tile[];
#pragma unroll
            for (int i = 0; i < 8; ++i) tile[turned(c.page_shift, dch * 8 + i, place / 4)] = w4[i];
            __syncthreads();
            const int n16 = (P * D) >> 4;
            for (int ch = threadIdx.x; ch < n16; ch += (P / 4) * (D / 8))
                __builtin_nontemporal_store(*(const v4i*)&tile[turned(c.page_shift, ch >> (c.page_shift - 4), (ch & (P / 16 - 1)) * 4)], (v4i*)codes + ch);
            return;
        }
        const bool all = place >= it.lo && place + 4 <= it.hi;
        if (!all && grown && place < it.lo) {                   // earlier tokens of this quad first
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                unsigned* at = (unsigned*)(col + (i << c.page_shift));
                const unsigned keep = place + 4 <= it.lo ? 0xffffffffu : (1u << (8 * (it.lo - place))) - 1u, w0 = *at;
                *at = (recode4<E5M2>(w0, down) & keep) | (w0 & ~keep);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint8_t* at = col + (i << c.page_shift);
            if (all) *(unsigned*)at = w4[i];
            else {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (place + u >= it.lo && place + u < it.hi) at[u] = (uint8_t)(w4[i] >> (8 * u));
            }
        }
    }
}

template <int D, bool E5M2>
__global__ void __launch_bounds__(1024)
kv_read_kernel(CacheView c, Rows k, Rows v, Spans s, int pages_per_seq)
{
    PageItem it;
    if (!find_item(c, s, pages_per_seq, it)) return;
    const Rows& dst = it.kv ? v : k;
    const uint8_t* codes = (it.kv ? c.v_codes : c.k_codes) + ((it.slab * D) << c.page_shift);
    char* row0 = dst.data + it.b * dst.stride_batch + it.h * dst.stride_head;
    const int P = 1 << c.page_shift;
    if (threadIdx.x >= (P / 4) * (D / 8)) return;
    const float sc = __int_as_float((int)(it.kv ? c.v_scales : c.k_scales)[it.slab] << 23);
    v4i out[4];
    if (it.kv == 0) {
        v2i w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            int place, dch;
            chunk_of<D>(0, c.page_shift, u, place, dch);
            w[u] = *(const v2i*)(codes + place * D + dch * 8);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const unsigned lo = (unsigned)w[u][0], hi = (unsigned)w[u][1];
            out[u] = v4i{decode2<E5M2, false>(lo, sc), decode2<E5M2, true>(lo, sc), decode2<E5M2, false>(hi, sc), decode2<E5M2, true>(hi, sc)};
        }
    } else {
        int place, dch;
        chunk_of<D>(1, c.page_shift, 0, place, dch);
        extern __shared__ __attribute__((aligned(16))) unsigned tile[];
        const int n16 = (P * D) >> 4;
        for (int ch = threadIdx.x; ch < n16; ch += (P / 4) * (D / 8))
            *(v4i*)&tile[turned(c.page_shift, ch >> (c.page_shift - 4), (ch & (P / 16 - 1)) * 4)] = ((const v4i*)codes)[ch];
        __syncthreads();
        unsigned w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = tile[turned(c.page_shift, dch * 8 + i, place / 4)];
        // the bytes of two channels side by side: positions 0 and 1, then 2 and 3
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const unsigned a = __builtin_amdgcn_perm(w[2 * p + 1], w[2 * p], 0x05010400u), b = __builtin_amdgcn_perm(w[2 * p + 1], w[2 * p], 0x07030602u);
            out[0][p] = decode2<E5M2, false>(a, sc);
            out[1][p] = decode2<E5M2, true>(a, sc);
            out[2][p] = decode2<E5M2, false>(b, sc);
            out[3][p] = decode2<E5M2, true>(b, sc);
        }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        int place, dch;
        chunk_of<D>(it.kv, c.page_shift, u, place, dch);
        if (place >= it.lo && place < it.hi)
            __builtin_nontemporal_store(out[u], (v4i*)(row0 + (int64_t)(it.first + place - it.start) * dst.stride_token + dch * 16));
    }
}

// One workgroup per page that N tokens can touch, kv head, and keys or values.
template <typename K>
static int launch_pages(K* const (&kernels)[2][2], const CacheView& c, const Rows& k, const Rows& v, const Spans& s, hipStream_t stream)
{
    const int P = 1 << c.page_shift;
    const int64_t pages = std::min((int64_t)((s.N + P - 2) >> c.page_shift) + 1, (int64_t)c.max_pages);
    if (pages == 0) return DMA_OK_;
    const int threads = std::max(64, (P / 4) * (c.D / 8));
    const int64_t per_page = (int64_t)c.Hkv * 2;
    if (pages > (int64_t)0x7fffffff / per_page || s.B > (int64_t)0x7fffffff / (per_page * pages)) return DMA_ERR_UNSUPPORTED_;
    const int64_t blocks = per_page * pages * s.B;
    if (blocks * threads > 0xffffffffLL) return DMA_ERR_UNSUPPORTED_;       // what a launch may hold
    return launch_lds(kernels[c.D == 128][c.e5m2], dim3((unsigned)blocks), dim3(threads), P * c.D, stream, c, k, v, s, (int)pages);
}

int launch_kv_write(const CacheView& c, const Rows& k, const Rows& v, const Spans& s, hipStream_t stream)
{
    using F = void(CacheView, Rows, Rows, Spans, int);
    F* const kernels[2][2] = {{kv_write_kernel<64, false>, kv_write_kernel<64, true>}, {kv_write_kernel<128, false>, kv_write_kernel<128, true>}};
    return launch_pages<F>(kernels, c, k, v, s, stream);
}

int launch_kv_read(const CacheView& c, const Rows& k, const Rows& v, const Spans& s, hipStream_t stream)
{
    using F = void(CacheView, Rows, Rows, Spans, int);
    F* const kernels[2][2] = {{kv_read_kernel<64, false>, kv_read_kernel<64, true>}, {kv_read_kernel<128, false>, kv_read_kernel<128, true>}};
    return launch_pages<F>(kernels, c, k, v, s, stream);
}

}  // namespace dma
