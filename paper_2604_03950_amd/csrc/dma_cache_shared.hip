// Attention over the paged 8-bit cache for sequences that share a prefix, which is read once for all of them.
//
// softmax(q k^T) v over keys that lie in parts joins from the parts' maxima, weights and sums: m = max m_i, l = sum l_i 2^(m_i - m),
// o = sum o_i 2^(m_i - m), out = o / l.  The shared part of a group (its positions below S = shared / 64 * 64, whole steps) is visited with
// the rows of all its sequences in tiles of 128: a step's codes are read and decoded once for 128 rows, as for a piece of a prompt
// (many_steps).  What a sequence has behind it is visited with its own rows, as for single tokens (few_rows).  One launch does both: the
// first is bound by matrix and vector work, the second by the bytes of the cache, and workgroups of both kinds share the CUs.  A second one
// joins.  Nothing here knows how long the sequences are until it runs: each workgroup finds its part of the work by itself.
#include "dma_cache_few.hpp"
#include "dma_cache_many.hpp"
#include <algorithm>

namespace dma {

constexpr int GROUPS_LDS = 512;              // groups whose bounds are kept in LDS
constexpr int ROWS_MANY = 128;
constexpr int WAVES = 4;

struct SharedArgs {
    CacheAttnArgs a;         // pieces and split: of what the sequences have to themselves
    Groups g;
    int rows_per_seq;        // query rows of a kv head and sequence: N * G
    float* pieces;           // of the prefixes: per workgroup [128][D] sums, [128] maxima, [128] weights
    int2* split;             // per item (kv head, row tile): the first piece and how many
    int64_t max_pieces;
    int resident;            // workgroups that the chip holds
};

struct Bounds {
    int lo, hi;              // sequences
    int steps;               // that they share
};
DMA_DEV int shared_steps(const SharedArgs& x, int shared) { return max(min(shared, x.a.capacity), 0) / STEP; }
DMA_DEV Bounds bounds_of(const SharedArgs& x, int g)
{
    Bounds r;
    r.lo = min(max(x.g.first[g], 0), x.a.s.B);
    r.hi = min(max(x.g.first[g + 1], r.lo), x.a.s.B);
    r.steps = shared_steps(x, x.g.shared[g]);
    return r;
}
// Items of the groups lie in order; this many at most before those of group g, whose first sequence is lo.
DMA_DEV int64_t tiles_before(const SharedArgs& x, int g, int lo) { return (int64_t)lo * x.rows_per_seq / ROWS_MANY + g; }

// The group of sequence b: the last one that does not begin behind it.  first(g): where group g begins.
template <typename F>
DMA_DEV int group_of(const F& first, int n, int b)
{
    int lo = 0, hi = n;                      // the answer + 1 is in [lo, hi]
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (first(mid) <= b) lo = mid + 1;
        else hi = mid;
    }
    return lo > 0 && b < first(lo) ? lo - 1 : -1;
}

// What a sequence has to itself begins where its group's shared part ends.
struct OwnBehindPrefix {
    static constexpr bool ON = true;
    const SharedArgs& x;
    const int* first;        // in LDS, where there are few groups
    const int* steps;
    DMA_DEV SeqInfo seq(const CacheAttnArgs& a, int b) const
    {
        SeqInfo q = seq_of(a, b);
        if (x.g.n <= GROUPS_LDS) {
            const int g = group_of([&](int i) { return first[i]; }, x.g.n, b);
            q.own = g < 0 ? 0 : steps[g];
        } else {
            const int g = group_of([&](int i) { return x.g.first[i]; }, x.g.n, b);
            q.own = g < 0 ? 0 : shared_steps(x, x.g.shared[g]);
        }
        return q;
    }
};

DMA_DEV int wave_scan(int x)                 // the sum up to and with this lane's
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);       // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);       // row_bcast:15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// One workgroup's part of the prefixes: 128 rows of a group, some of their steps, into piece `piece`.
template <int D, bool E5M2, bool UNI>
DMA_DEV void prefix_part(const SharedArgs& x, const ManyLds<D>& lds, int (&ends)[4][WAVES], const Bounds& g, int h, int tile, int part, int parts, int64_t piece)
{
    const CacheAttnArgs& a = x.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int64_t all_rows = (int64_t)(g.hi - g.lo) * x.rows_per_seq;
    const int rows = (int)min(all_rows - (int64_t)tile * ROWS_MANY, (int64_t)ROWS_MANY), my_rows = min(rows - wave * 32, 32);
    // ---- this lane's row: sequence, token and head
    const int64_t r = min((int64_t)tile * ROWS_MANY + wave * 32 + col, all_rows - 1);
    const int b = g.lo + (int)((unsigned)r / (unsigned)x.rows_per_seq), in_seq = (int)((unsigned)r % (unsigned)x.rows_per_seq);
    const int tok = in_seq / a.G;
    v8bf qf[D / 16];
    {
        const char* qp = a.q.data + b * a.q.stride_batch + (h * a.G + in_seq - tok * a.G) * a.q.stride_head + tok * a.q.stride_token;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const v8bf*)(qp + (ks * 16 + half * 8) * 2);
    }
    const SeqInfo sq = seq_of(a, b);
    const bool exists = tok < sq.n && col < my_rows;
    // ---- what is visible.  Rows that do not exist have no say in it
    const int64_t at = (int64_t)sq.start + tok;
    ManyRows view;
    view.my_rows = my_rows;
    view.vis_hi = exists ? cut_position(at) : -1;
    view.vis_lo = exists && a.window ? cut_position(at - a.window + 1) : 0;
    auto wave_max = [](int v) {
        for (int s = 16; s; s >>= 1) v = max(v, __shfl_xor(v, s));
        return __builtin_amdgcn_readfirstlane(v);
    };
    view.all_hi = -wave_max(exists ? -view.vis_hi : -POS_MAX);
    view.some_hi = wave_max(view.vis_hi);
    view.all_lo = wave_max(view.vis_lo);
    view.some_lo = -wave_max(exists ? -view.vis_lo : -POS_MAX);
    if (lane == 0) {
        ends[0][wave] = view.all_hi;
        ends[1][wave] = view.some_hi;
        ends[2][wave] = view.all_lo;
        ends[3][wave] = view.some_lo;
    }
    __syncthreads();
    view.wg_hi = min(min(ends[0][0], ends[0][1]), min(ends[0][2], ends[0][3]));
    view.any_hi = max(max(ends[1][0], ends[1][1]), max(ends[1][2], ends[1][3]));
    view.wg_lo = max(max(ends[2][0], ends[2][1]), max(ends[2][2], ends[2][3]));
    view.any_lo = min(min(ends[3][0], ends[3][1]), min(ends[3][2], ends[3][3]));
    view.wg_hi = __builtin_amdgcn_readfirstlane(view.wg_hi);
    view.any_hi = __builtin_amdgcn_readfirstlane(view.any_hi);
    view.wg_lo = __builtin_amdgcn_readfirstlane(view.wg_lo);
    view.any_lo = __builtin_amdgcn_readfirstlane(view.any_lo);
    // ---- the steps: of the shared ones, those that a row sees
    const int hi = min(view.any_hi + 1, g.steps * STEP), lo = min(view.any_lo, hi);
    StepRange range;
    range.base = 0;
    range.first = lo / STEP;
    range.sink_steps = (min(a.sinks, hi) + STEP - 1) / STEP;
    if (range.sink_steps >= range.first) range.sink_steps = range.first = 0;
    range.steps = range.sink_steps + (hi + STEP - 1) / STEP - range.first;
    const int begin = (int)((int64_t)range.steps * part / parts), end = (int)((int64_t)range.steps * (part + 1) / parts);
    v16f o[D / 32];
    float m, l;
    many_steps<D, E5M2, WAVES, UNI>(a, lds, g.lo, h, range, begin, end, view, qf, o, m, l);
    if (col >= my_rows) return;
    l = cross_half_sum(l);
    float* p = x.pieces + piece * (ROWS_MANY * (D + 2));
    const int rr = wave * 32 + col;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *(v4f*)(p + rr * D + dt * 32 + 8 * q + 4 * half) = v4f{o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]};
    if (half == 0) {
        p[ROWS_MANY * D + rr] = m;
        p[ROWS_MANY * D + ROWS_MANY + rr] = l;
    }
}

// What a step costs a workgroup: 64 positions for 128 rows of a prefix, and for one row tile of a sequence's own.
constexpr int COST_MANY = 3, COST_FEW = 2;

// Rows of a sequence: tiles of 16 * MT.
template <int D, bool E5M2, int MT, bool UNI>
__global__ void __launch_bounds__(64 * WAVES, 2)
cache_shared_kernel(SharedArgs x)
{
    using Few = FewLds<D, MT, WAVES>;
    using Many = ManyLds<D>;
    constexpr size_t FEW = sizeof(typename Few::O) + sizeof(typename Few::Q) + sizeof(typename Few::Ml), MANY = sizeof(typename Many::K) + sizeof(typename Many::V);
    __shared__ __attribute__((aligned(16))) char buffer[FEW > MANY ? FEW : MANY];
    __shared__ int odd[4], ends[4][WAVES], first[GROUPS_LDS + 1], steps[GROUPS_LDS];
    const CacheAttnArgs& a = x.a;
    if (x.g.n <= GROUPS_LDS) {
        for (int g = threadIdx.x; g <= x.g.n; g += 64 * WAVES) first[g] = x.g.first[g];
        for (int g = threadIdx.x; g < x.g.n; g += 64 * WAVES) steps[g] = shared_steps(x, x.g.shared[g]);
        __syncthreads();
    }
    const int lane = threadIdx.x & 63;
    const Few few = {*(typename Few::O*)buffer, *(typename Few::Ml*)(buffer + sizeof(typename Few::O) + sizeof(typename Few::Q)), *(typename Few::Q*)(buffer + sizeof(typename Few::O))};
    const OwnBehindPrefix own = {x, first, steps};

    auto role = [&](int own_units, unsigned& block, unsigned& blocks) {
        // ---- how much work the prefixes are
        auto load = [&](int g, Bounds& r, int& tiles, int& visited) {
            r = Bounds{0, 0, 0};
            if (g < x.g.n) r = bounds_of(x, g);
            tiles = (int)(((int64_t)(r.hi - r.lo) * x.rows_per_seq + ROWS_MANY - 1) / ROWS_MANY);
            // under a window the steps differ from tile to tile: about as many as one token visits
            visited = a.window ? min(r.steps, (int)min((int64_t)r.steps, (a.sinks + (int64_t)a.window + a.s.N) / STEP + 3)) : r.steps;
        };
        Bounds r;
        int tiles, visited;
        int64_t total = 0;
        for (int base = 0; base < x.g.n; base += 64) {
            load(base + lane, r, tiles, visited);
            int64_t w = (int64_t)tiles * visited;
            for (int s = 32; s; s >>= 1) w += __shfl_xor(w, s);
            total += w;
        }
        total *= a.c.Hkv;
        // ---- which of the workgroups do which, by what the steps cost
        const int64_t few_cost = ((int64_t)own_units << a.unit_shift) * COST_FEW, many_cost = total * COST_MANY;
        int few_blocks = x.resident;
        if (total) few_blocks = min(max((int)((double)x.resident * few_cost / (few_cost + many_cost)) / 8 * 8, 8), x.resident - 8);
        block = blockIdx.x;
        blocks = few_blocks;
        if (total == 0 || (int)blockIdx.x < few_blocks) return (int)blockIdx.x < few_blocks;
        // ---- pieces of the prefixes' items: equal parts of each
        const int share = (int)max((total + (x.resident - few_blocks) - 1) / (x.resident - few_blocks), (int64_t)2);
        auto pieces_of = [&] { return (int)min((int64_t)tiles * a.c.Hkv * ((visited + share - 1) / share), (int64_t)1 << 24); };
        int all = 0;
        for (int base = 0; base < x.g.n; base += 64) {
            if (x.g.n > 64 || base > 0) load(base + lane, r, tiles, visited);
            all += __builtin_amdgcn_readlane(wave_scan(pieces_of()), 63);
            if (all < 0) return false;                              // (bounds that decrease)
        }
        // workgroups next to each other in the list on the same XCD: they read the same keys
        const int per = (all + 7) / 8, p = blockIdx.x - few_blocks, at = p % 8 * per + p / 8;
        if (p / 8 >= per || at >= all) return false;
        int before = 0;
        for (int base = 0; base < x.g.n; base += 64) {
            if (x.g.n > 64) load(base + lane, r, tiles, visited);
            const int upto = wave_scan(pieces_of()), sum = __builtin_amdgcn_readlane(upto, 63);
            if (at < before + sum) {
                const int who = __builtin_ctzll(__ballot(before + upto > at));
                Bounds mine;
                mine.lo = __builtin_amdgcn_readlane(r.lo, who);
                mine.hi = __builtin_amdgcn_readlane(r.hi, who);
                mine.steps = __builtin_amdgcn_readlane(r.steps, who);
                const int n_tiles = __builtin_amdgcn_readlane(tiles, who), parts = (__builtin_amdgcn_readlane(visited, who) + share - 1) / share;
                const int first_piece = before + __builtin_amdgcn_readlane(upto, who) - n_tiles * a.c.Hkv * parts;
                const int i = at - first_piece, tile = i % n_tiles, part = i / n_tiles % parts, h = i / n_tiles / parts;
                const int item = h * n_tiles + tile;
                const int64_t piece = (int64_t)first_piece + item * parts + part;
                if (i < 0 || h >= a.c.Hkv || piece < 0 || piece >= x.max_pieces) return false;      // (bounds that decrease)
                if (part == 0 && threadIdx.x == 0) x.split[(tiles_before(x, base + who, mine.lo)) * a.c.Hkv + item] = make_int2(first_piece + item * parts, parts);
                const Many many = {*(typename Many::K*)buffer, *(typename Many::V*)(buffer + sizeof(typename Many::K)), odd};
                prefix_part<D, E5M2, UNI>(x, many, ends, mine, h, tile, part, parts, piece);
                return false;
            }
            before += sum;
        }
        return false;
    };
    few_rows<D, E5M2, MT, WAVES, false, UNI>(a, few, own, role);
}

// Joins the pieces of the prefix and of a sequence's own: a workgroup per sequence, kv head and 4 of its rows; threads over channels (4 each),
// rows and pieces.
template <int D, int ROWS>
__global__ void __launch_bounds__(512)
cache_shared_join_kernel(SharedArgs x)
{
    constexpr int CH = D / 4, PG = 512 / (4 * CH), U = 4;
    const CacheAttnArgs& a = x.a;
    const int h = blockIdx.x % (unsigned)a.c.Hkv, b = blockIdx.x / (unsigned)a.c.Hkv;
    const SeqInfo sq = seq_of(a, b);
    const int rows = sq.n * a.G, r0 = blockIdx.y * 4, rr = threadIdx.x / CH % 4, ch = threadIdx.x % CH, pg = threadIdx.x / (4 * CH);
    if (r0 >= rows) return;
    const int row = min(r0 + rr, rows - 1);
    // ---- where the pieces are
    const int g = group_of([&](int i) { return x.g.first[i]; }, x.g.n, b);
    int own_first, own_n, many_first = 0, many_n = 0, many_row = 0;
    {
        const int2 sp = a.split[((int64_t)b * a.c.Hkv + h) * a.row_tiles + row / ROWS];
        own_first = sp.x;
        own_n = sp.y - sp.x + 1;
    }
    if (g >= 0) {
        const Bounds r = bounds_of(x, g);
        if (r.steps > 0) {
            const int64_t in_group = (int64_t)(b - r.lo) * x.rows_per_seq + row;
            const int n_tiles = (int)(((int64_t)(r.hi - r.lo) * x.rows_per_seq + ROWS_MANY - 1) / ROWS_MANY);
            const int2 sp = x.split[tiles_before(x, g, r.lo) * a.c.Hkv + h * n_tiles + in_group / ROWS_MANY];
            // (within the workspace whatever the bounds of the groups say)
            many_first = max(sp.x, 0);
            many_n = (int)min((int64_t)max(sp.y, 0), max(x.max_pieces - many_first, (int64_t)0));
            many_row = (int)(in_group % ROWS_MANY);
        }
    }
    v4f o = {0.f, 0.f, 0.f, 0.f};
    float m = M_NONE, l = 0.f;
    const int n = own_n + many_n;
    for (int w = pg; w < n; w += PG * U) {
        float m2[U], l2[U];
        v4f y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = w + u * PG;
            m2[u] = M_NONE;
            l2[u] = 0.f;
            y[u] = v4f{0.f, 0.f, 0.f, 0.f};
            if (i < n) {
                const bool mine = i < own_n;
                const float* p = mine ? a.pieces + (int64_t)(own_first + i) * (ROWS * (D + 2)) : x.pieces + (int64_t)(many_first + i - own_n) * (ROWS_MANY * (D + 2));
                const int at = mine ? row % ROWS : many_row, all = mine ? ROWS : ROWS_MANY;
                m2[u] = p[all * D + at];
                l2[u] = p[all * D + all + at];
                y[u] = *(const v4f*)(p + at * D + ch * 4);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (w + u * PG >= n) break;
            const float up = fmaxf(m, m2[u]);
            const float f1 = __builtin_amdgcn_exp2f((m - up) * a.scale), f2 = __builtin_amdgcn_exp2f((m2[u] - up) * a.scale);
            m = up;
            l = l * f1 + l2[u] * f2;
            o = o * f1 + y[u] * f2;
        }
    }
    __shared__ v4f os[PG][4][CH];
    __shared__ float ms[PG][4], ls[PG][4];
    os[pg][rr][ch] = o;
    if (ch == 0) {
        ms[pg][rr] = m;
        ls[pg][rr] = l;
    }
    __syncthreads();
    if (pg || r0 + rr >= rows) return;
    for (int k = 1; k < min(PG, n); ++k) {
        const float m2 = ms[k][rr], up = fmaxf(m, m2);
        const float f1 = __builtin_amdgcn_exp2f((m - up) * a.scale), f2 = __builtin_amdgcn_exp2f((m2 - up) * a.scale);
        m = up;
        l = l * f1 + ls[k][rr] * f2;
        o = o * f1 + os[k][rr][ch] * f2;
    }
    const int i = row / a.G;
    char* op = a.out.data + b * a.out.stride_batch + (h * a.G + row - i * a.G) * a.out.stride_head + i * a.out.stride_token;
    const v4f y = o * (l == 0.f ? 0.f : 1.f / l);
    *(v2i*)(op + ch * 8) = v2i{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
}

// ---------------------------------------------------------------------------------------------------------------- host
// Sizes of a call: row tiles of a sequence, items of both kinds and their pieces at most.
struct SharedSizes {
    int mt, resident;
    int64_t tiles, few_items, few_pieces, many_items, many_pieces, blocks;
    size_t bytes;
    bool fits;
};
static SharedSizes sizes_of(const CacheView& c, int B, int G, int N, int n_groups)
{
    SharedSizes z;
    const int64_t rows = (int64_t)N * G;
    z.mt = rows <= 16 ? 1 : 2;
    z.tiles = (rows + 16 * z.mt - 1) / (16 * z.mt);
    z.resident = (2 * cache_cus() + 15) / 16 * 16;
    z.few_items = (int64_t)B * c.Hkv * z.tiles;
    z.few_pieces = z.resident + z.few_items;
    z.many_items = ((int64_t)B * rows / ROWS_MANY + n_groups + 1) * c.Hkv;
    z.many_pieces = z.resident + (B * rows / ROWS_MANY + std::min(n_groups, B) + 1) * (int64_t)c.Hkv;
    z.blocks = z.resident + z.many_pieces;
    z.bytes = (size_t)((z.few_pieces * 16 * z.mt + z.many_pieces * ROWS_MANY) * (c.D + 2) * 4 + (z.few_items + z.many_items) * 8);
    z.fits = z.blocks * 256 <= 0xffffffffLL && (int64_t)B * c.Hkv * ((rows + 3) / 4) <= 0xffffffffLL / 512 && z.few_pieces < 1 << 30;
    return z;
}

// Whether sequences are taken together at all.
static bool together(const SharedSizes& z, int G, int N, int n_groups) { return n_groups > 0 && (int64_t)N * G <= ROWS_MANY && z.fits; }

size_t cache_attn_shared_workspace(const CacheView& c, int B, int Hq, int N, int n_groups, int window, int sinks)
{
    const SharedSizes z = sizes_of(c, B, Hq / c.Hkv, N, n_groups);
    return together(z, Hq / c.Hkv, N, n_groups) ? z.bytes : cache_attn_workspace(c, B, Hq, N, window, sinks);
}

template <int D, bool E5M2, int MT>
static int launch_shared(const SharedArgs& x, const SharedSizes& z, hipStream_t stream)
{
    const dim3 grid((unsigned)z.blocks), block(64 * WAVES);
    const int rc = x.a.c.page_shift >= 6 ? launch(cache_shared_kernel<D, E5M2, MT, true>, grid, block, stream, x) : launch(cache_shared_kernel<D, E5M2, MT, false>, grid, block, stream, x);
    if (rc != DMA_OK_) return rc;
    return launch(cache_shared_join_kernel<D, 16 * MT>, dim3((unsigned)(x.a.s.B * x.a.c.Hkv), (unsigned)((x.rows_per_seq + 3) / 4)), dim3(512), stream, x);
}

int launch_cache_attn_shared(const CacheView& c, const Rows& q, const Rows& out, const Spans& s, int Hq, const Groups& groups, int window, int sinks,
                             void* workspace, hipStream_t stream)
{
    const SharedSizes z = sizes_of(c, s.B, Hq / c.Hkv, s.N, groups.n);
    if (!together(z, Hq / c.Hkv, s.N, groups.n)) return launch_cache_attn(c, q, out, s, Hq, window, sinks, workspace, stream);
    SharedArgs x = {};
    CacheAttnArgs& a = x.a;
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
    a.row_tiles = (int)z.tiles;
    // the units of the line are counted in 31 bits
    while (z.few_items * ((a.capacity / STEP >> a.unit_shift) + 2) > 0x7fffffff) ++a.unit_shift;
    x.g = groups;
    x.rows_per_seq = s.N * a.G;
    x.resident = z.resident;
    x.max_pieces = z.many_pieces;
    a.pieces = (float*)workspace;
    x.pieces = a.pieces + z.few_pieces * 16 * z.mt * (c.D + 2);
    a.split = (int2*)(x.pieces + z.many_pieces * ROWS_MANY * (c.D + 2));
    x.split = a.split + z.few_items;
    auto pick = [&](auto D, auto F) { return z.mt == 1 ? launch_shared<D, F != 0, 1>(x, z, stream) : launch_shared<D, F != 0, 2>(x, z, stream); };
    if (c.D == 128) return c.e5m2 ? pick(IC<128>{}, IC<1>{}) : pick(IC<128>{}, IC<0>{});
    return c.e5m2 ? pick(IC<64>{}, IC<1>{}) : pick(IC<64>{}, IC<0>{});
}

}  // namespace dma
