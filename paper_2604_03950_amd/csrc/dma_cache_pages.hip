// Pages that several sequences hold: rows of the page table that take over others' entries (fork), free pages handed out and shared ones
// copied before they are written (reserve), pages in use brought to the first places (compact).
//
// The work on the table and on refs is integers in memory that fits the caches: bound by latency.  What is copied is whole pages, which
// lie in one piece on each side (all kv heads of them): bound by memory.
#include "dma_internal.hpp"
#include "dma_device.hpp"
#include <algorithm>

namespace dma {

// ---------------------------------------------------------------------------------------------------------------- fork
// A column of the new table depends on that column of the old one alone: a workgroup holds some columns of all rows in LDS, so that rows can
// take over each other's entries in place, and counts there how many rows take over each: what row r named is named (that - 1) times more.
// One atomic at most per entry that is not taken over exactly once, instead of one for each that goes and one for each that comes.
//
// 8 rows of 16 entries: 2.7 us, bound by latency (three trips to memory and LDS one behind the other).  256 rows of up to 2048, of which every eighth
// takes the place of seven: 16 us for 2.1 MB of table; 7 of them are a count read and written for each of 314 000 pages in random places, 9 the table, of
// whose lines of 128 bytes a workgroup has 16: 29 MB are read for 4.2.  (With an
// atomic for each entry that goes or comes, and no LDS, 39 call to call, now 18; with all loads of a workgroup of 1024 in flight at once 21.)
__global__ void __launch_bounds__(256)
kv_fork_kernel(CacheView c, int* table, int* refs, int B, int cols_shift, const int* src, const int* length)
{
    extern __shared__ int2 tile[];           // an entry, and how often it is taken over
    const int cols = 1 << cols_shift, n = B << cols_shift;
    for (int j0 = blockIdx.x << cols_shift; j0 < c.max_pages; j0 += gridDim.x << cols_shift) {
        for (int e = threadIdx.x; e < n; e += 256) {
            const int j = j0 + (e & (cols - 1));
            tile[e] = make_int2(j < c.max_pages ? table[(int64_t)(e >> cols_shift) * c.max_pages + j] : -1, 0);
        }
        __syncthreads();
        for (int e = threadIdx.x; e < n; e += 256) {
            const int b = e >> cols_shift, j = j0 + (e & (cols - 1)), from = src[b];
            if (j >= c.max_pages) continue;
            const int keep = length ? length[b] : 0x7fffffff;
            int page = -1;
            if ((unsigned)from < (unsigned)B && (int64_t)j << c.page_shift < keep) {
                int2& taken = tile[(from << cols_shift) + (e & (cols - 1))];
                page = taken.x;
                if ((unsigned)page >= c.page_limit) page = -1;
                else atomicAdd(&taken.y, 1);
            }
            if (page != tile[e].x) table[(int64_t)b * c.max_pages + j] = page;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < n; e += 256) {
            const int2 was = tile[e];
            if (was.y == 1 || (unsigned)was.x >= c.page_limit) continue;
            // A count of one is this entry's own: every other one that named the page has been taken off it, and nobody else changes it.
            if (refs[was.x] == 1) refs[was.x] = was.y;
            else atomicAdd(&refs[was.x], was.y - 1);
        }
        __syncthreads();
    }
}

int launch_kv_fork(const CacheView& c, int* refs, int B, const int* src, const int* length, hipStream_t stream)
{
    if (c.max_pages == 0) return DMA_OK_;
    int shift = 4;
    while (shift && (B << shift) > FORK_ROWS_MAX) --shift;              // 64 KiB of LDS
    // ... and fewer columns where that leaves CUs without any (256 rows of 2048 entries: 18 us call to call, with 16 columns always 27)
    while (shift > 2 && (c.max_pages >> shift) < 512) --shift;
    const int blocks = std::min((c.max_pages + (1 << shift) - 1) >> shift, 4096);
    return launch_lds(kv_fork_kernel, dim3(blocks), dim3(256), (size_t)(B << shift) * 8, stream, c, (int*)c.page_table, refs, B, shift, src, length);
}

// --------------------------------------------------------------------------------------------------------- page copies
// A slice of a page's codes (the keys' slices, then the values', each side `bytes`) from page `from` to page `to`, by a workgroup of 256 threads:
// 16 bytes per thread and turn, four in flight.  Stores pass the caches by, which hold less than what is copied; loads as well where each page is
// read once (ONCE; where samples of one prompt part, all of them copy one page).  1000 pages of 131 KB: both 45 us = 5.8 TB/s, stores alone 46.4,
// neither 51.6.
constexpr int SLICE = 16384;
template <bool ONCE>
DMA_DEV void copy_slice(const CacheView& c, int64_t bytes, int from, int to, int slice)
{
    const int side = (int)((bytes + SLICE - 1) / SLICE);
    const uint8_t* codes = slice < side ? c.k_codes : c.v_codes;
    const int64_t first = (int64_t)(slice < side ? slice : slice - side) * SLICE, end = min(first + SLICE, bytes);
    const uint8_t* src = codes + from * bytes;
    uint8_t* dst = (uint8_t*)codes + to * bytes;
    v4i w[4];
    if (end - first == SLICE) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const v4i* at = (const v4i*)(src + first + threadIdx.x * 16 + u * 4096);
            w[u] = ONCE ? __builtin_nontemporal_load(at) : *at;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) __builtin_nontemporal_store(w[u], (v4i*)(dst + first + threadIdx.x * 16 + u * 4096));
    } else {
        for (int64_t at = first + threadIdx.x * 16; at < end; at += 4096) *(v4i*)(dst + at) = *(const v4i*)(src + at);
    }
}
DMA_DEV_CONSTEXPR int64_t slices_of(int64_t bytes) { return 2 * ((bytes + SLICE - 1) / SLICE); }

// Where thread t of 1024 stands among those before it: the sum of `mine` over them, and over all in `total`.
DMA_DEV int scan_1024(int mine, int* wave_sums, int& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = mine;
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);       // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);       // row_bcast:15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    __syncthreads();                                                      // the sums of the scan before have been read
    if (lane == 63) wave_sums[wave] = x;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        const int s = wave_sums[w];
        if (w < wave) before += s;
        total += s;
    }
    return before + x - mine;
}

// ------------------------------------------------------------------------------------------------------------- reserve
constexpr int NOT_GIVEN = -1, GIVEN_NEW = -2;      // in the workspace, per entry; otherwise the page that the sequence leaves

// One workgroup: entries in order, 1024 at a time; free pages are looked for as far as they are needed, in a ring in LDS.  Which page an entry gets
// follows from the entries before it alone, so that equal calls give equal tables: sums over the workgroup instead of atomics.
//
// Bound by latency: start, entry, refs of the page, sums, refs of the free pages, one behind the other.  64 sequences with a token each: 3.6 us;
// 13 with up to 4100 tokens in pages of 32: 6.5; 256 with one each: 4.3.  Pages are looked at from the first on, 4096 per turn of 1.2 us: where the first 130 000 of
// 131 072 are used, both kernels take 48 us call to call, 8.5 where the first 8000 hold a free one.
__global__ void __launch_bounds__(1024)
kv_reserve_kernel(CacheView c, int* table, int* refs, Spans s, int pages_per_seq, int* missing, int* left)
{
    constexpr int RING = 8192;
    __shared__ int ring[RING], wave_sums[16];
    for (int b = threadIdx.x; b < s.B; b += 1024) missing[b] = 0;
    __syncthreads();
    const int64_t entries = (int64_t)s.B * pages_per_seq, capacity = (int64_t)c.max_pages << c.page_shift;
    int64_t looked = 0;                            // pages whose refs have been looked at
    unsigned head = 0, fill = 0;                   // free pages given and found
    for (int64_t first = 0; first < entries; first += 1024) {
        const int64_t e = first + threadIdx.x;
        bool wants = false;
        int b = 0, old = GIVEN_NEW;
        int64_t at = 0;
        if (e < entries) {
            b = (int)((unsigned)e / (unsigned)pages_per_seq);
            const int start = s.start[b], n = s.n_tokens ? min(max(s.n_tokens[b], 0), s.N) : s.N;
            const int64_t j = (start >> c.page_shift) + ((unsigned)e - (unsigned)b * (unsigned)pages_per_seq);
            if (start >= 0 && n > 0 && j << c.page_shift < min((int64_t)start + n, capacity)) {
                at = (int64_t)b * c.max_pages + j;
                const int page = table[at];
                wants = (unsigned)page >= c.page_limit;
                if (!wants && refs[page] > 1) {
                    wants = true;
                    old = page;
                }
            }
        }
        int asked;
        const int rank = scan_1024(wants, wave_sums, asked);
        while ((int)(fill - head) < asked && looked < c.num_pages) {
            const int64_t p = looked + threadIdx.x * 4;
            bool is_free[4];
            int mine = 0, found;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                is_free[u] = p + u < c.num_pages && refs[p + u] == 0;
                mine += is_free[u];
            }
            unsigned to = fill + scan_1024(mine, wave_sums, found);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (is_free[u]) ring[to++ % RING] = (int)(p + u);
            fill += found;
            looked += 4096;
        }
        __syncthreads();
        bool given = false;
        if (wants) {
            given = rank < (int)(fill - head);
            if (given) {
                const int page = ring[(head + rank) % RING];
                table[at] = page;
                refs[page] = 1;
            } else {
                atomicAdd(&missing[b], 1);
            }
        }
        if (e < entries) left[e] = given ? old : NOT_GIVEN;
        head += min((unsigned)asked, fill - head);
        __syncthreads();                           // before the ring is filled again
    }
}

// What became of the entries: shared pages are one holder poorer, the earlier tokens in them are copied, other new pages hold nothing.
// blockIdx.y: a slice of the copies; the first has the rest as well.
//
// Workgroups for every sequence, whether it copies or not, as the host knows no counts: one without work ends behind a load.  64 sequences, 56 of which
// copy a page of 128 KiB (7 MB written): 5.0 us, bound by latency; 256 that copy one of 512 KiB (134 MB written, all
// from one page): 26.6 us = 5.0 TB/s of stores, bound by memory.
__global__ void __launch_bounds__(256)
kv_part_kernel(CacheView c, const int* table, int* refs, Spans s, int pages_per_seq, const int* left)
{
    const int64_t bytes = (int64_t)c.Hkv * c.D << c.page_shift;
    for (int b = blockIdx.x; b < s.B; b += gridDim.x) {
        const int start = s.start[b], j0 = start >> c.page_shift;
        const int* l = left + (int64_t)b * pages_per_seq;
        const int* row = table + (int64_t)b * c.max_pages;
        const bool part = start >= 0 && (start & ((1 << c.page_shift) - 1)) != 0;
        if (blockIdx.y == 0) {
            // entries times kv heads over the threads
            const int step = max(256 / c.Hkv, 1), k0 = threadIdx.x / c.Hkv, h0 = c.Hkv > 256 ? threadIdx.x : threadIdx.x - k0 * c.Hkv;
            for (int k = c.Hkv > 256 ? 0 : k0; k < pages_per_seq && (c.Hkv > 256 || k0 < step); k += step) {
                const int old = l[k];
                if (old == NOT_GIVEN) continue;
                if (old >= 0 && h0 == 0) atomicAdd(&refs[old], -1);
                const bool copied = old >= 0 && k == 0 && part;
                const int64_t to = (int64_t)row[j0 + k] * c.Hkv, from = copied ? (int64_t)old * c.Hkv : 0;
                for (int h = h0; h < c.Hkv; h += 256) {
                    c.k_scales[to + h] = copied ? c.k_scales[from + h] : 255;
                    c.v_scales[to + h] = copied ? c.v_scales[from + h] : 255;
                }
            }
        }
        const int old = l[0];
        if (old < 0 || !part) continue;
        const int to = row[j0];
        for (int64_t slice = blockIdx.y; slice < slices_of(bytes); slice += gridDim.y) copy_slice<false>(c, bytes, old, to, (int)slice);
    }
}

int64_t reserve_pages(const CacheView& c, int N) { return std::min((int64_t)((N + (1 << c.page_shift) - 2) >> c.page_shift) + 1, (int64_t)c.max_pages); }

int launch_kv_reserve(const CacheView& c, int* refs, const Spans& s, int* missing, int* workspace, hipStream_t stream)
{
    const int pages = (int)reserve_pages(c, s.N);
    const int rc = launch(kv_reserve_kernel, dim3(1), dim3(1024), stream, c, (int*)c.page_table, refs, s, pages, missing, workspace);
    if (rc != DMA_OK_ || pages == 0) return rc;
    const int64_t slices = std::min<int64_t>(slices_of((int64_t)c.Hkv * c.D << c.page_shift), 64);
    return launch(kv_part_kernel, dim3(std::min(s.B, 8192), (unsigned)slices), dim3(256), stream, c, c.page_table, refs, s, pages, (const int*)workspace);
}

// ------------------------------------------------------------------------------------------------------------- compact
// The workspace: how many moves, then (from, to) of each.
struct Moves {
    int count, pad;
    int2 move[1];
};
size_t compact_workspace(const CacheView& c) { return 8 + 8 * (size_t)(c.num_pages / 2); }

// One workgroup: counts, then lists free pages below the count and used ones from there on.  In order, so that equal calls give equal tables.
// Bound by latency: 300 pages 3.6 us, 4096 pages 6.1, 131 072 (call to call, nothing to move) 107.
__global__ void __launch_bounds__(1024)
kv_compact_plan_kernel(CacheView c, const int* refs, int* used_out, int* moved, Moves* moves)
{
    __shared__ int wave_sums[16];
    int mine = 0, used;
    for (int64_t p = threadIdx.x; p < c.num_pages; p += 1024) mine += refs[p] > 0;
    scan_1024(mine, wave_sums, used);
    int holes = 0, movers = 0;
    for (int64_t first = 0; first < c.num_pages; first += 4096) {
        const int64_t p = first + threadIdx.x * 4;
        bool in_use[4];
        int hole = 0, mover = 0, found;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            in_use[u] = p + u < c.num_pages && refs[p + u] > 0;
            hole += p + u < used && !in_use[u];
            mover += p + u >= used && in_use[u];
        }
        int at = holes + scan_1024(hole, wave_sums, found);
        holes += found;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (p + u < used && !in_use[u]) moves->move[at++].y = (int)(p + u);
        // (holds for the pages below `used`, all of them before any that moves)
        at = movers + scan_1024(mover, wave_sums, found);
        movers += found;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (p + u >= c.num_pages) continue;
            int to = in_use[u] ? (int)(p + u) : -1;
            if (p + u >= used && in_use[u]) {
                to = moves->move[at].y;
                moves->move[at++].x = (int)(p + u);
            }
            moved[p + u] = to;
        }
    }
    if (threadIdx.x == 0) {
        *used_out = used;
        moves->count = movers;
    }
}

// Copies the pages that move, and renames them in the table, which nothing else of it reads.  1000 pages of 131 KB out of 4096, and 256 rows of the table:
// 46 us = 5.7 TB/s read and written, a large copy's rate; 300 pages of which 40 move: 3.5.
__global__ void __launch_bounds__(256)
kv_compact_kernel(CacheView c, int* table, int* refs, int64_t entries, const int* moved, const Moves* moves)
{
    const int count = moves->count;
    const int64_t bytes = (int64_t)c.Hkv * c.D << c.page_shift, slices = slices_of(bytes), all = slices * count;
    for (int64_t i = blockIdx.x; i < all; i += gridDim.x) {
        const int64_t which = i / slices;
        const int part = (int)(i - which * slices);
        const int2 m = moves->move[which];
        copy_slice<true>(c, bytes, m.x, m.y, part);
        if (part == 0) {
            for (int h = threadIdx.x; h < c.Hkv; h += 256) {
                c.k_scales[(int64_t)m.y * c.Hkv + h] = c.k_scales[(int64_t)m.x * c.Hkv + h];
                c.v_scales[(int64_t)m.y * c.Hkv + h] = c.v_scales[(int64_t)m.x * c.Hkv + h];
            }
            if (threadIdx.x == 0) {
                refs[m.y] = refs[m.x];
                refs[m.x] = 0;
            }
        }
    }
    if (count == 0) return;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < entries; e += (int64_t)gridDim.x * 256) {
        const int page = table[e];
        if ((unsigned)page < c.page_limit) table[e] = moved[page];
    }
}

int launch_kv_compact(const CacheView& c, int* refs, int B, int* used, int* moved, void* workspace, hipStream_t stream)
{
    const int rc = launch(kv_compact_plan_kernel, dim3(1), dim3(1024), stream, c, (const int*)refs, used, moved, (Moves*)workspace);
    if (rc != DMA_OK_) return rc;
    // a slice for each workgroup, as far as the host knows how many there can be
    const int64_t slices = c.num_pages / 2 * slices_of((int64_t)c.Hkv * c.D << c.page_shift), blocks = std::min<int64_t>(std::max<int64_t>(slices, 1024), 16384);
    return launch(kv_compact_kernel, dim3((unsigned)blocks), dim3(256), stream, c, (int*)c.page_table, refs, (int64_t)B * c.max_pages, (const int*)moved, (const Moves*)workspace);
}

}  // namespace dma
