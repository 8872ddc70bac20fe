// Attention of drafted tokens that form a tree over the paged cache (include/alora_tree.h).
//
// The rows of a sequence read the same context, so a workgroup takes a tile of them and loads every cached row once for all; what a row
// sees of the drafts, which lie behind the context, a mask says.  The contexts are cut into parts of one length, found on the device
// from all lengths of the call (their sum is not known on the host), so that workgroups have equal work however ragged the lengths are.
#include <algorithm>
#include "alora_tree.h"
#include "alora_listed.h"

namespace alora {

// A tile of a sequence's rows, for the kernel that combines its parts: numbers first, first + step, ...
struct TreeTile {
    int row0, rows, parts, first, step, pad[3];
};

// What a workgroup (of each K/V head) is for.
struct TreeItem {
    int row0, rows;             // the tile's rows
    int seq, ctx, end;          // end: of the drafts that lie in the table
    int lo, hi, part;           // places of the sequence it reads; number of its part's sums, -1: the whole tile
};

struct TreeArgs {
    ListArgs list;
    const int32_t *offsets, *context;
    const uint32_t *mask;       // [T][2 * words]
    int words, tile_rows;       // rows of a tile
    int lg_unit;
    int places;                 // workgroups per K/V head that the chip holds at once, two to a compute unit (of the vector kernel's with eight columns one: their turns are two)
    int least_units;            // of a part
    int max_tiles, max_items, max_parts;      // the workspace has room for
    int *found;                 // tiles, items
    TreeTile *tiles;
    TreeItem *items;            // of more than ALONE sequences
};

constexpr int LG_UNIT = 5;      // parts are counted in units of 32 positions; of 64 where a table has more than 2^29, so that a sequence's are 2^24 at most, which floats count

constexpr int ALONE = 64;       // sequences up to which every wavefront finds its item by itself
constexpr int CLASSES = 4;      // of parts by their length

constexpr int CUTS = 5;
// What a call costs in units (32 positions of a tile), by what was measured: a workgroup's start, and a part's sums.
constexpr float START = 7.f, PART = 7.f;

struct TreeSeq {
    int r0, n, ctx, places, tiles, units;
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeArgs &a, int s)
{
    const ListArgs &g = a.list;
    TreeSeq q = {0, 0, 0, 0, 0, 0};
    if (s < g.n_seqs) {
        const int cap = g.max_blocks * g.bs;
        q.r0 = min(max(a.offsets[s], 0), g.T);
        q.n = min(max(a.offsets[s + 1], q.r0), g.T) - q.r0;
        q.ctx = min(max(a.context[s], 0), cap);
        q.places = min(q.ctx + min(q.n, 64 * a.words), cap);
        q.tiles = (q.n + a.tile_rows - 1) / a.tile_rows;
        q.units = (q.places + (1 << a.lg_unit) - 1) >> a.lg_unit;
    }
    return q;
}

// Units of a part: no part is longer.  Found from all sequences, NW wavefronts together (for_each calls a function for each sequence of a thread); 0: there are no tiles, or more
// than ascending offsets give.
template <int NW>
struct CutScratch {
    float sums[3 + 3 * CUTS][NW];
};
template <int NW, class ForEach>
__device__ __forceinline__ int units_of_parts(const TreeArgs &a, CutScratch<NW> *scr, ForEach for_each)
{
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // N sums, every third one a maximum: over a thread's sequences -> over all
    auto over_all = [&](auto &x, int at) {
        constexpr int N = sizeof(x) / sizeof(float);
        auto over_lanes = [&](float y, bool largest) {
            y = largest ? __int_as_float(max_upto64(__float_as_int(y))) : sum_upto64(y);
            return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(y), 63));
        };
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = over_lanes(x[i], i % 3 == 2);
            if (NW > 1 && lane == 0) scr->sums[at + i][w] = x[i];
        }
        if (NW == 1) return;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = over_lanes(lane < NW ? scr->sums[at + i][lane] : 0.f, i % 3 == 2);
    };
    // Units of all tiles, tiles, the longest.
    float all[3] = {0.f, 0.f, 0.f};
    for_each([&](const TreeSeq &x) {
        all[0] += (float)x.tiles * (float)x.units;
        all[1] += (float)x.tiles;
        all[2] = fmaxf(all[2], x.tiles ? (float)x.units : 0.f);
    });
    over_all(all, 0);
    const float total = all[0], tiles = all[1], most = fmaxf(all[2], 1.f);
    if (tiles == 0.f || tiles > (float)a.max_tiles) return 0;
    // (Reciprocals: an IEEE division is 15 instructions, and up to ALONE sequences every workgroup does this before its first copy.)
    auto over = [](float x, float y) { return x * __builtin_amdgcn_rcpf(y); };
    const float places = (float)a.places, share = over(total, places), room = places - tiles, half = .5f * places - tiles;
    float units = most;
    if (half >= 1.f) {
        // Few tiles: as many parts as fit the chip in one turn, or, of short contexts, half of it, a workgroup to each compute unit (a tile's last part may be
        // short: one more for each).  us, 32/8 heads, when every wavefront had columns of its own, 128, 256, 384, 512, 768 workgroups: 13 rows at 9000 positions 25.2, 21.1, 24.9, 24.8, 24.7, at 32000 59.7, 39.4,
        // 40.4, 37.9, 47.6, 4 x 13 rows at 16000 106, 63.5, 62.5, 53.7, 68.6; 64/8 heads, 64 rows at 64000 387, 212, 209, 181, 204.
        // Two workgroups on a compute unit take 1.8 times as long for a position as one by itself, and leave four units' worth of parts more.  us, half | one turn: 13 rows at 14000
        // 21.5 | 23.6, at 20000 25.7 | 28.0, at 32000 35.5 | 35.5, 8 x 8 rows at 3000 30.8 | 26.2, 16 x 8 at 1000 27.3 | 22.6.
        auto units_for = [&](float n) { return fmaxf(fminf(ceilf(over(total, n)), most), (float)a.least_units); };
        const float two = units_for(room), one = units_for(half);
        units = one < 1.8f * two + 4.f ? one : two;
    } else {
        // Many: the best of whole tiles, an equal share for every place of the chip or two thirds of it, as many parts as fit in one turn or in two.
        float cut[CUTS] = {most, share, share * (2.f / 3), over(total, room), over(total, 2.f * places - tiles)};
        float of[3 * CUTS] = {}, one_over[CUTS];      // items, those of them that are parts, the longest
#pragma unroll
        for (int i = 0; i < CUTS; ++i) {
            cut[i] = cut[i] > 0.f ? fmaxf(fminf(ceilf(cut[i]), most), (float)a.least_units) : most;
            one_over[i] = __builtin_amdgcn_rcpf(cut[i]);
        }
        for_each([&](const TreeSeq &x) {
#pragma unroll
            for (int i = 0; i < CUTS; ++i) {
                float parts = fmaxf(ceilf((float)x.units * one_over[i] - 1e-3f), 1.f);
                if (fmaf(parts, cut[i], -(float)x.units) < 0.f) parts += 1.f;      // (exact: the parts' sums need room)
                const float n = parts * (float)x.tiles;
                of[3 * i] += n;
                of[3 * i + 1] += parts > 1.f ? n : 0.f;
                of[3 * i + 2] = fmaxf(of[3 * i + 2], x.tiles ? over((float)x.units, parts) : 0.f);
            }
        });
        over_all(of, 3);
        float best = 3.0e38f;
#pragma unroll
        for (int i = 0; i < CUTS; ++i) {
            // In units: as many turns as the chip takes, or its places filled by the longest first; a start for each turn; what parts leave and are combined from.
            const float m = of[3 * i + 2], filled = over(of[3 * i], places), turns = ceilf(filled - 1e-3f);
            const float span = fminf(turns * m, fmaxf(m, fminf(share, filled * m) + m * (1.f / 3))), cost = span + START * turns + over(PART * of[3 * i + 1], places);
            if (cost < best && of[3 * i + 1] <= (float)a.max_parts) best = cost, units = cut[i];      // (whole tiles have no parts)
        }
    }
    return max(1, (int)fminf(units, 1.0e9f));
}

// A sequence's parts are equal, none longer than `per`; the longest start first (in quarters of per).
struct TreeCut {
    int parts, size, kind;      // units of a part (the last one's may be fewer), class
};
__device__ __forceinline__ TreeCut tree_cut(const TreeSeq &q, int per)
{
    TreeCut c;
    c.parts = max(1, (q.units + per - 1) / per);
    c.size = (q.units + c.parts - 1) / c.parts;
    c.kind = min(CLASSES - 1, (int)((float)(per - c.size) * (float)CLASSES * __builtin_amdgcn_rcpf((float)per)));
    return c;
}
// Item `i` of a sequence (tiles of one part next to each other: they read the same rows), whose parts' numbers begin at `part_at`.
__device__ __forceinline__ TreeItem tree_item(const TreeArgs &a, int s, const TreeSeq &q, const TreeCut &c, int part_at, int i)
{
    const int part = i / q.tiles, tile = i - part * q.tiles;
    const long long lo = (long long)part * c.size << a.lg_unit, hi = lo + ((long long)c.size << a.lg_unit);
    return {q.r0 + tile * a.tile_rows, min(a.tile_rows, q.n - tile * a.tile_rows), s, q.ctx, q.places, (int)min(lo, (long long)q.places), (int)min(hi, (long long)q.places), c.parts > 1 ? part_at + i : -1};
}

// Which tile and part workgroup `item` (of one K/V head) is for; false: none.
__device__ __forceinline__ bool find_item(const TreeArgs &a, int item, int hk, TreeItem &it)
{
    const int lane = threadIdx.x & 63;
    if (a.list.n_seqs > ALONE) {
        const int n = a.found[1];
        const TreeItem x = a.items[item];
        int *const to = (int *)&it, *const from = (int *)&x;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(TreeItem) / 4); ++i) to[i] = __builtin_amdgcn_readfirstlane(from[i]);
        return item < n && it.part < a.max_parts;
    }
    // The same sums, in the same order, in every wavefront of the call.
    const TreeSeq q = tree_seq(a, lane);
    const int per = units_of_parts<1>(a, (CutScratch<1> *)nullptr, [&](auto f) { f(q); });
    if (per == 0) {
        if (item == 0 && hk == 0 && threadIdx.x == 0) a.found[0] = 0;
        return false;
    }
    const TreeCut c = tree_cut(q, per);
    const int items = q.tiles * c.parts, tiles_upto = sum_upto64(q.tiles), numbered = c.parts > 1 ? items : 0, part_at = sum_upto64(numbered) - numbered;
    int at = 0, all = 0;
#pragma unroll
    for (int i = 0; i < CLASSES; ++i) {
        const int mine = c.kind == i ? items : 0, upto = sum_upto64(mine);
        if (c.kind == i) at = all + upto - mine;
        all += __builtin_amdgcn_readlane(upto, 63);
    }
    if (item == 0 && hk == 0 && threadIdx.x == 63) a.found[0] = tiles_upto;
    const bool here = item >= at && item < at + items;
    TreeItem mine = {};
    if (here) {
        mine = tree_item(a, lane, q, c, part_at, item - at);
        const int tile = item - at;             // (of part 0)
        if (hk == 0 && threadIdx.x < 64 && tile < q.tiles) a.tiles[tiles_upto - q.tiles + tile] = {mine.row0, mine.rows, c.parts, part_at + tile, q.tiles, {}};
    }
    const unsigned long long who = __builtin_amdgcn_ballot_w64(here);
    if (!who) return false;
    int *const to = (int *)&it, *const from = (int *)&mine;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(TreeItem) / 4); ++i) to[i] = __builtin_amdgcn_readlane(from[i], (int)__builtin_ctzll(who));
    return it.part < a.max_parts;
}

// The same for more sequences, once for all workgroups, by one: what each item is, in the workspace.  (Done by every workgroup itself it took 6 to 7 us of each.)
template <int THREADS>
__global__ __launch_bounds__(THREADS) void tree_plan_kernel(TreeArgs a)
{
    constexpr int NW = THREADS / 64;
    __shared__ CutScratch<NW> scr;
    __shared__ int counts[NW][CLASSES + 2];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n_seqs = a.list.n_seqs;
    const TreeSeq q0 = tree_seq(a, tid);
    auto for_each = [&](auto f) {
        f(q0);
        for (int s = tid + THREADS; s < n_seqs; s += THREADS) f(tree_seq(a, s));
    };
    const int per = units_of_parts<NW>(a, &scr, for_each);
    if (per == 0) {
        if (tid == 0) a.found[0] = a.found[1] = 0;
        return;
    }
    // Where a class's items begin, and the tiles, and the parts' numbers: `begin` of the sequences before.
    int begin[CLASSES + 2] = {}, n[CLASSES] = {};
    for_each([&](const TreeSeq &x) {
        const TreeCut c = tree_cut(x, per);
#pragma unroll
        for (int i = 0; i < CLASSES; ++i) n[i] += c.kind == i ? x.tiles * c.parts : 0;
    });
#pragma unroll
    for (int i = 0; i < CLASSES; ++i) {
        const int u = sum_upto64(n[i]);
        if (lane == 63) counts[w][i] = u;
    }
    __syncthreads();
    int upto = 0;
#pragma unroll
    for (int i = 0; i < CLASSES; ++i) {
        begin[i] = upto;
        upto += __builtin_amdgcn_readlane(sum_upto64(lane < NW ? counts[lane][i] : 0), 63);
    }
    if (tid == 0) a.found[1] = min(upto, a.max_items);
    for (int s0 = 0; s0 < n_seqs; s0 += THREADS) {
        const TreeSeq q = s0 ? tree_seq(a, s0 + tid) : q0;
        const TreeCut c = tree_cut(q, per);
        const int items = q.tiles * c.parts;
        int mine[CLASSES + 2], sum[CLASSES + 2];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < CLASSES + 2; ++i) {
            mine[i] = i == CLASSES ? q.tiles : i > CLASSES ? (c.parts > 1 ? items : 0) : c.kind == i ? items : 0;
            sum[i] = sum_upto64(mine[i]);
            if (lane == 63) counts[w][i] = sum[i];
        }
        __syncthreads();
        int at = 0, tile_at = 0, part_at = 0;
#pragma unroll
        for (int i = 0; i < CLASSES + 2; ++i) {
            const int of_waves = sum_upto64(lane < NW ? counts[lane][i] : 0), here = begin[i] + (w ? __builtin_amdgcn_readlane(of_waves, w - 1) : 0) + sum[i] - mine[i];
            begin[i] += __builtin_amdgcn_readlane(of_waves, 63);
            if (i == CLASSES) tile_at = here;
            else if (i > CLASSES) part_at = here;
            else if (c.kind == i) at = here;
        }
        // a few items by the sequence's thread, many by its wavefront
        auto put = [&](int s, const TreeSeq &q, const TreeCut &c, int at, int tile_at, int part_at, int i) {
            const TreeItem it = tree_item(a, s, q, c, part_at, i);
            if (at + i < a.max_items) a.items[at + i] = it;
            if (i < q.tiles && tile_at + i < a.max_tiles) a.tiles[tile_at + i] = {it.row0, it.rows, c.parts, part_at + i, q.tiles, {}};
        };
        const bool many = items > 8;
        if (!many)
            for (int i = 0; i < items; ++i) put(s0 + tid, q, c, at, tile_at, part_at, i);
        for (unsigned long long todo = __builtin_amdgcn_ballot_w64(many); todo; todo &= todo - 1) {
            const int from = (int)__builtin_ctzll(todo);
            auto its = [&](int x) { return __builtin_amdgcn_readlane(x, from); };
            const TreeSeq theirs = {its(q.r0), its(q.n), its(q.ctx), its(q.places), its(q.tiles), its(q.units)};
            const TreeCut cut = {its(c.parts), its(c.size), its(c.kind)};
            for (int i = lane; i < its(items); i += 64) put(s0 + 64 * w + from, theirs, cut, its(at), its(tile_at), its(part_at), i);
        }
    }
    if (tid == 0) a.found[0] = min(begin[CLASSES], a.max_tiles);
}

// Rows of no sequence: zeros.  Done by the workgroups of a K/V head behind those for items, 64 rows of the call each (as many as there may be in a batch
// that is padded to a fixed size), at most MOST_CLEARING.
constexpr int MOST_CLEARING = 256;
template <int D, bool BF16, int NW>
__device__ __forceinline__ void clear_rows(const TreeArgs &a, int hk, int number, int of)
{
    const ListArgs &g = a.list;
    const int begin = g.n_seqs ? min(max(a.offsets[0], 0), g.T) : 0, end = g.n_seqs ? min(max(a.offsets[g.n_seqs], begin), g.T) : 0;
    const int chunks = (D << g.lg_g) * (BF16 ? 2 : 4) / 16;
    const size_t width = (size_t)g.Hq * D * (BF16 ? 2 : 4);
    auto clear = [&](int t0, int t1) {
        for (long long i = (long long)number * (64 * NW) + threadIdx.x; i < (long long)(t1 - t0) * chunks; i += (long long)of * (64 * NW))
            *(u32x4 *)((char *)g.out + (t0 + i / chunks) * width + ((size_t)hk * chunks + i % chunks) * 16) = (u32x4){0u, 0u, 0u, 0u};
    };
    clear(0, begin);
    clear(end, g.T);
}

// C columns: C >> lg_g rows of a sequence.
template <int D, int C>
__global__ __launch_bounds__(256) void tree_vector_kernel(TreeArgs a)
{
    __shared__ VectorScratch<C, D> scr;
    __shared__ uint32_t bits[C][2 * ALORA_MAX_TREE_WORDS];
    const ListArgs &g = a.list;
    const int hk = (int)blockIdx.x % g.Hkv, item = (int)blockIdx.x / g.Hkv, tid = threadIdx.x;
    if (item >= a.max_items) return clear_rows<D, false, 4>(a, hk, item - a.max_items, (int)(gridDim.x / g.Hkv) - a.max_items);
    TreeItem it;
    if (!find_item(a, item, hk, it)) return;
    const int G = 1 << g.lg_g;
    if (tid < 2 * a.words * it.rows) bits[tid / (2 * a.words)][tid % (2 * a.words)] = a.mask[(size_t)it.row0 * 2 * a.words + tid];
    __syncthreads();
    const int32_t *bt = g.bt + (size_t)it.seq * g.max_blocks;
    const auto column_at = [&](int c) { return (((long long)it.row0 + (c >> g.lg_g)) * g.Hq + hk * G + (c & (G - 1))) * D; };
    read_list_vector<D, C>(
        g, hk, scr, it.lo, it.hi, it.ctx,
        [&](int v) { return slot_at(g, bt, v / g.bs, v % g.bs); },
        [&](int c, int v) { return v < it.ctx || (bits[c >> g.lg_g][(v - it.ctx) >> 5] >> ((v - it.ctx) & 31) & 1u); },
        [&](int c) { return c >> g.lg_g < it.rows ? column_at(c) : -1ll; },
        [&](int c, int d, float M, float L, float o) {
            if (c >> g.lg_g >= it.rows) return;
            if (it.part >= 0) {
                const size_t at = ((size_t)it.part * g.Hkv + hk) * C + c;
                if (d == 0) *(f32x2 *)(g.ml + 2 * at) = (f32x2){M, L};
                g.o[at * D + d] = o;
                return;
            }
            ((float *)g.out)[column_at(c) + d] = L == 0.f ? 0.f : o / L;
        });
}

// 32 columns a wavefront: 128 >> lg_g rows of a sequence.  What bounds it: with wide trees matrix and vector unit in turn (48 sequences of up to 64 drafts over up to 16000
// positions, 64 / 8 heads, 318 GFLOP: 631 us with the parts combined, 0.50 PFLOP/s of products that count; the matrix unit is busy for 39 % of the cycles, the vector unit for 50; 64 x 64 rows over
// 8192, 32 / 8 heads, whose tiles are full, 950 us, 0.57 of 0.86 made), with many narrow ones memory (64 x 8 rows over 8192, 2.1 GB: 346 us, 6.2 TB/s), with one latency (13 rows over 9001, 15.4 us: to find its
// part 1.9, slots 1.2, first tiles 1.5, the rest two tiles at a time).  The weights are whole, as for selected blocks: the error against 64 bits is that of the result's rounding.
// Rounded once to bf16, with two thirds of the products, they cost as much again as that rounding; us, rounded once | whole: 13 rows at 9000 positions 16.4 | 16.8, 64 x 8 rows
// at 8192 347 | 345, 64 x 16 349 | 360, 64 x 24 390 | 468, 64 x 64 779 | 956.  (The rest's products behind or between the others', placed by hand: within 1 %.)
constexpr int WAVES = 4;
template <int D, bool ONCE, bool SHARE>
__global__ __launch_bounds__(64 * WAVES, 2) void tree_matrix_kernel(TreeArgs a)
{
    __shared__ MatrixTiles<D, WAVES, 32, 512 / D, 2, 2048> lds;      // 64 KiB of tiles: two workgroups share a CU's LDS
    const ListArgs &g = a.list;
    const int hk = (int)blockIdx.x % g.Hkv, item = (int)blockIdx.x / g.Hkv;
    if (item >= a.max_items) return clear_rows<D, true, WAVES>(a, hk, item - a.max_items, (int)(gridDim.x / g.Hkv) - a.max_items);
    TreeItem it;
    if (!find_item(a, item, hk, it)) return;
    const int32_t *bt = g.bt + (size_t)it.seq * g.max_blocks;
    const int columns = it.rows << g.lg_g;
    const bool share = SHARE && columns <= 32 * WAVES / 2;
    const int col = 32 * (((int)threadIdx.x >> 6) & (share ? WAVES / 2 - 1 : WAVES - 1)) + ((int)threadIdx.x & 31), row = it.row0 + (min(col, columns - 1) >> g.lg_g);
    const uint32_t *bits = a.mask + (size_t)row * 2 * a.words;
    const size_t at = ((size_t)row * g.Hq + ((size_t)hk << g.lg_g) + (col & ((1 << g.lg_g) - 1))) * D;
    read_list_matrix<ONCE, SHARE>(
        g, hk, lds, it.lo, it.hi, it.ctx, columns, share,
        [&](int v) { return slot_at(g, bt, v / g.bs, v % g.bs); },
        [&](int place) {               // the row's bits of drafts place - ctx .. + 31; what lies in front of them is seen
            const int from = place - it.ctx, i = from >> 5, s = from & 31;
            const uint32_t x = i < 0 ? 0xffffffffu : i < 2 * a.words ? bits[i] : 0u, y = i + 1 < 2 * a.words ? bits[i + 1] : 0u;
            return s ? x >> s | y << (32 - s) : x;
        },
        at, at, it.part >= 0 ? (long long)it.part * g.Hkv + hk : -1ll, 32 * WAVES);
}

// One wavefront per column of a tile that has parts, of a tile's with many tiles several.  Bound by the latency of tile, sums and store where there are few (4.5 us for 31 parts of one tile);
// 48 sequences of up to 64 rows 32 us for 17 MB of sums, with waves that wait for 57 % of their time.
template <int D, bool BF16, int AHEAD>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, int columns)
{
    const ListArgs &g = a.list;
    const int hk = (int)blockIdx.x % g.Hkv, tile = (int)blockIdx.x / g.Hkv;
    const int n = a.found[0];
    const TreeTile t = a.tiles[tile];      // (both loads at once: there is room for as many as workgroups)
    if (tile >= n || t.parts <= 1 || (long long)t.first + (long long)(t.parts - 1) * t.step >= a.max_parts) return;
    for (int c = (int)blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); c >> g.lg_g < t.rows; c += (int)gridDim.y * 4)
        combine_parts<D, BF16, AHEAD>(g, (size_t)t.first * g.Hkv + hk, (size_t)t.step * g.Hkv, t.parts, columns, c,
                                      ((size_t)(t.row0 + (c >> g.lg_g)) * g.Hq + ((size_t)hk << g.lg_g) + (c & ((1 << g.lg_g) - 1))) * D);
}

// ---- host ---------------------------------------------------------------------------------------
// How a call is cut: columns of a tile, the most tiles and items (tile, part) of a K/V head there can be, and where the workspace's arrays lie.
struct TreePlan {
    bool matrix;                // instructions; else vector arithmetic
    int columns, tile_rows, places;
    long long tiles, items, parts;
    size_t tiles_at, items_at, ml_at, o_at, bytes;
};
static TreePlan plan_tree(const alora_attn_dims *d)
{
    TreePlan p;
    const int G = d->n_q_heads / d->n_kv_heads;
    p.matrix = d->dtype == ALORA_BF16;
    p.columns = p.matrix ? 32 * WAVES : std::max(4, G);      // (fp32, heads of 128, 2, 4, 8 columns, us: 30 rows at 4000 positions, 4 sequences, 4/2 heads, 72, 61, 109, 16 at 8000, 8 sequences, 8/4 heads, 258, 204, 425)
    p.tile_rows = p.columns / G;
    p.places = std::max(1, 512 / d->n_kv_heads);
    p.tiles = d->n_tokens / p.tile_rows + std::min(d->n_seqs, d->n_tokens);      // (a sequence's last tile may not be full)
    p.items = p.tiles + 2ll * p.places + 2;                                      // sum of ceil(units / per) over tiles, see units_of_parts
    p.parts = std::min(p.items, 4ll * p.places + 8);                             // (few tiles have as many as there are places at most; of many tiles' cuts none with more is taken)
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    p.tiles_at = 256;
    p.items_at = p.tiles_at + up((size_t)p.tiles * sizeof(TreeTile));
    p.ml_at = p.items_at + (d->n_seqs > ALONE ? up((size_t)p.items * sizeof(TreeItem)) : 0);
    p.o_at = p.ml_at + up((size_t)p.parts * d->n_kv_heads * p.columns * 8);
    p.bytes = p.o_at + (size_t)p.parts * d->n_kv_heads * p.columns * d->head_dim * 4;
    return p;
}

static int check_tree(const alora_attn_dims *d, int words)
{
    const int st = check_attention(d);
    if (st) return st;
    if (words < 1 || words > ALORA_MAX_TREE_WORDS || d->n_seqs > 1 << 20) return ALORA_ESHAPE;
    if ((long long)d->max_blocks * d->block_size > 1 << 30) return ALORA_ESHAPE;
    if ((plan_tree(d).items + MOST_CLEARING) * d->n_kv_heads >= 1 << 24) return ALORA_ESHAPE;      // (workgroups of 256: a grid holds fewer than 2^32 threads)
    return ALORA_OK;
}

}  // namespace alora

using namespace alora;

extern "C" {

int alora_tree_attention_workspace_bytes(const alora_attn_dims *dims, int32_t mask_words, size_t *out_bytes)
{
    if (!out_bytes) return ALORA_EINVAL;
    const int st = check_tree(dims, mask_words);
    if (st) return st;
    *out_bytes = dims->n_tokens ? plan_tree(dims).bytes : 0;
    return ALORA_OK;
}

int alora_tree_attention(const void *q, const void *k_cache, const void *v_cache, const int32_t *block_tables, const int32_t *row_offsets,
                         const int32_t *context_lens, const uint64_t *tree_mask, int32_t mask_words, void *out, const alora_attn_dims *dims,
                         void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int st = check_tree(dims, mask_words);
    if (st) return st;
    if (dims->n_tokens == 0) return ALORA_OK;
    const TreePlan p = plan_tree(dims);
    if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < p.bytes) return ALORA_EWORKSPACE;
    if (!q || !k_cache || !v_cache || no_table(dims, block_tables) || !row_offsets || (dims->n_seqs && !context_lens) || !tree_mask || !out) return ALORA_EINVAL;
    if (((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)out) & 15 || (uintptr_t)tree_mask & 7) return ALORA_EINVAL;
    if (((uintptr_t)block_tables | (uintptr_t)row_offsets | (uintptr_t)context_lens) & 3) return ALORA_EINVAL;
    TreeArgs a;
    a.list = list_args(dims, q, k_cache, v_cache, block_tables, out);
    a.list.ml = (float *)((char *)workspace + p.ml_at);
    a.list.o = (float *)((char *)workspace + p.o_at);
    a.offsets = row_offsets; a.context = context_lens;
    a.mask = (const uint32_t *)tree_mask; a.words = mask_words;
    a.tile_rows = p.tile_rows; a.lg_unit = LG_UNIT + ((long long)dims->max_blocks * dims->block_size > 1 << 29); a.places = p.places; a.least_units = p.matrix ? 8 : 4;      // (fp32, 5 trees over up to 700 positions, eight columns: 2 units 22.2 us, 4 20.7, 8 23.8)
    a.max_tiles = (int)p.tiles; a.max_items = (int)p.items; a.max_parts = (int)p.parts;
    a.found = (int *)workspace;
    a.tiles = (TreeTile *)((char *)workspace + p.tiles_at);
    a.items = (TreeItem *)((char *)workspace + p.items_at);
    const bool bf16 = dims->dtype == ALORA_BF16;
    // About 8192 workgroups combine parts: most tiles of a call with many have none (32 for each tile: 1000 sequences 72 us for nothing, now 5).  us, 2048, 8192, 32768
    // workgroups: 64 x 4 rows at 300 positions 24.2, 25.7, 28.1, 16 x 8 at 4000 56.7, 56.9, 56.6; 48 ragged sequences of up to 64 rows 547, 525, 521.
    const int clearing = std::min(MOST_CLEARING, 1 + dims->n_tokens / 64);
    // (no tiles: fewer rows than one holds, and no sequence they could be of)
    const long long merging = p.tiles * dims->n_kv_heads;
    const dim3 grid((unsigned)((p.items + clearing) * dims->n_kv_heads)), merge((unsigned)merging, (unsigned)std::clamp(8192 / std::max(1ll, merging), 1ll, p.columns / 4ll));
    const auto go = [&](auto kernel, auto combine) {
        // (us, 256 | 1024 threads: 65 sequences of 300 positions 33.6 | 36.5, 256 of 1000 197 | 199, 1000 of 300 294 | 291, 3000 of 200 626 | 613)
        if (dims->n_seqs > 512) launch_kernel(tree_plan_kernel<1024>, dim3(1), dim3(1024), 0, (hipStream_t)hip_stream, a);
        else if (dims->n_seqs > ALONE) launch_kernel(tree_plan_kernel<256>, dim3(1), dim3(256), 0, (hipStream_t)hip_stream, a);
        launch_kernel(kernel, grid, dim3(64 * WAVES), 0, (hipStream_t)hip_stream, a);
        if (merging) launch_kernel(combine, merge, dim3(256), 0, (hipStream_t)hip_stream, a, p.columns);
    };
    // Non-temporal copies where a sequence brings one tile on average: then its context is read once.  us, ordinary | non-temporal, 32/8 heads: 13 rows at 9000
    // positions 21.0 | 19.5, at 128000 118 | 113, 64 x 8 rows at 8192 381 | 352, 64 x 24 475 | 462, 64 x 32 537 | 525, 64 x 40 (two tiles) 865 | 876, 16 x 8 at 4000 54.4 | 58.5;
    // 48 of up to 64 rows, 64/8 heads, 633 | 676.
    const long long columns = (long long)dims->n_tokens * (dims->n_q_heads / dims->n_kv_heads);
    const bool once = columns <= 32ll * WAVES * dims->n_seqs;
    // Where half of the wavefronts have columns on average, the kernel that lets the other half take every second tile.  us, without | with: 13 rows at 2000
    // positions 15.7 | 15.3, at 9000 19.5 | 17.2, at 128000 113 | 101, 16 x 8 rows at 1000 24.6 | 22.8, 64 x 8 at 8192 352 | 346, 64 x 16 407 | 360.  (With wider
    // trees it loses: 64 x 40 876 | 884, 48 of up to 64 rows and 8 heads a group 676 | 681.)
    const bool share = columns <= 16ll * WAVES * dims->n_seqs;
    // Parts combined 16 at a time where a tile may have more than 16 of them (13 rows at 9001 positions 20.2 | 19.5 us; 16 x 8 rows at 4000, of fewer, 57.0 | 59.7).
    const bool many_parts = p.tiles <= p.places / 32;
    const auto choose = [&](auto head_dim) {
        constexpr int D = decltype(head_dim)::value;
        if (!bf16) p.columns == 4 ? go(tree_vector_kernel<D, 4>, tree_merge_kernel<D, false, 8>) : go(tree_vector_kernel<D, 8>, tree_merge_kernel<D, false, 8>);
        else if (share) many_parts ? go(tree_matrix_kernel<D, true, true>, tree_merge_kernel<D, true, 16>) : go(tree_matrix_kernel<D, true, true>, tree_merge_kernel<D, true, 8>);
        else once ? go(tree_matrix_kernel<D, true, false>, tree_merge_kernel<D, true, 8>) : go(tree_matrix_kernel<D, false, false>, tree_merge_kernel<D, true, 8>);
    };
    if (dims->head_dim == 128) choose(std::integral_constant<int, 128>{});
    else choose(std::integral_constant<int, 64>{});
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

}  // extern "C"
