// Attention of drafted tokens that form a tree over the paged cache (include/alora_tree.h).
//
// The rows of a sequence read the same context, so a workgroup takes a tile of them and loads every cached row once for all; what a row
// sees of the drafts, which lie behind the context, a mask says.  The contexts are cut into parts of one length, found on the device
// from all lengths of the call (their sum is not known on the host), so that workgroups have equal work however ragged the lengths are.
#include <algorithm>
#include <new>
#include "alora_tree.h"
#include "alora_listed.h"

namespace alora {

// A tile of a sequence's rows, for the kernel that combines its parts.
struct TreeTile {
    int row0, rows, parts, first, step, pad[3];
};

struct TreeArgs {
    ListArgs list;
    const int32_t *offsets, *context;
    const uint32_t *mask;       // [T][2 * words]
    int words, tile_rows;       // rows of a tile
    int places;                 // workgroups per K/V head that the chip holds at once
    int max_tiles, max_items;   // the workspace has room for (offsets that do not ascend may give more)
    int *n_tiles;
    TreeTile *tiles;
};

constexpr int UNIT = 32;        // positions that parts are counted in
constexpr int LEAST_UNITS = 8;  // of a part
constexpr int GOOD_UNITS = 12;

struct TreeItem {
    int row0, rows;             // the tile's rows
    int seq, ctx, drafts;       // drafts: those that lie in the table
    int lo, hi, parts, part_at; // places of the sequence this workgroup reads; number of its part's sums
};

constexpr int CLASSES = 4;      // of parts by their length

struct TreeScratch {
    float total[8][2];
    int sums[8][CLASSES + 1], found[8];
};

// Which tile and part workgroup `item` (of one K/V head, NW wavefronts) is for; false: none.  The same sums in every workgroup of the call.
// A sequence's parts are equal, none longer than `per`; the longest start first (in quarters of per): 48 contexts of 1000 to 16000, wide trees, in
// batch order ORDER_US.
template <int NW>
__device__ __forceinline__ bool find_item(const TreeArgs &a, int item, int hk, TreeScratch &scr, TreeItem &it)
{
    const ListArgs &g = a.list;
    constexpr int NT = 64 * NW;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, n_seqs = g.n_seqs;
    const long long cap = min((long long)g.max_blocks * g.bs, 0x7fffffffll);
    struct Seq { int r0, n, ctx, places, tiles, units; };
    auto seq_of = [&](int s) {
        Seq q = {0, 0, 0, 0, 0, 0};
        if (s < n_seqs) {
            q.r0 = min(max(a.offsets[s], 0), g.T);
            q.n = min(max(a.offsets[s + 1], q.r0), g.T) - q.r0;
            q.ctx = (int)min((long long)max(a.context[s], 0), cap);
            q.places = (int)min((long long)q.ctx + min(q.n, 64 * a.words), cap);
            q.tiles = (q.n + a.tile_rows - 1) / a.tile_rows;
            q.units = (q.places + UNIT - 1) / UNIT;
        }
        return q;
    };
    // all units of all tiles, and the tiles, in a fixed order
    Seq q = seq_of(tid);
    float mine = 0.f, mine_tiles = 0.f;
    for (int s = tid;; s += NT) {
        const Seq x = s == tid ? q : seq_of(s);
        mine += (float)x.tiles * (float)x.units;
        mine_tiles += (float)x.tiles;
        if (s + NT >= n_seqs) break;
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) mine += __shfl_xor(mine, off), mine_tiles += __shfl_xor(mine_tiles, off);
    if (lane == 0) scr.total[w][0] = mine, scr.total[w][1] = mine_tiles;
    if (tid == 0) scr.found[0] = -1;
    __syncthreads();
    float total = 0.f, tiles = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) total += scr.total[i][0], tiles += scr.total[i][1];
    // Units of a part.  Few tiles: as many workgroups as the chip holds at once (a tile's last part may be short: one more for each), of short contexts half as many,
    // one to a compute unit.  Many: one and a half times as many, the longest first.  us, 32/8 heads, 128, 256, 384, 512, 768 workgroups: 13 rows at 9000
    // positions 25.2, 21.1, 24.9, 24.8, 24.7, at 32000 59.7, 39.4, 40.4, 37.9, 47.6, 4 x 13 rows at 16000 106, 63.5, 62.5, 53.7, 68.6; 64/8 heads, 64 rows at
    // 64000 387, 212, 209, 181, 204.
    const float room = (float)a.places - tiles, half = (float)(a.places / 2) - tiles;
    float units = ceilf(total / ((float)a.places * 1.5f));
    if (2.f * tiles <= (float)a.places) units = ceilf(total / room);
    if (units < (float)GOOD_UNITS && half >= 1.f) units = ceilf(total / half);
    const int per = max(LEAST_UNITS, (int)fminf(units, 1.0e9f));
    auto parts_of = [&](const Seq &x) { return max(1, (x.units + per - 1) / per); };
    auto size_of = [&](const Seq &x, int parts) { return (x.units + parts - 1) / parts; };      // units of a part (the last one's may be fewer)
    auto class_of = [&](int size) { return min(CLASSES - 1, (int)((float)(per - size) * (float)CLASSES / (float)per)); };
    // where a class's items begin: one chunk of requests finds it with their own places, more of them ahead
    int begin[CLASSES + 1] = {};           // (the last: tiles)
    if (n_seqs > NT) {
        int count[CLASSES] = {};
        for (int s = tid; s < n_seqs; s += NT) {
            const Seq x = s == tid ? q : seq_of(s);
            const int parts = parts_of(x), c = class_of(size_of(x, parts));
#pragma unroll
            for (int i = 0; i < CLASSES; ++i) count[i] += c == i ? x.tiles * parts : 0;
        }
#pragma unroll
        for (int i = 0; i < CLASSES; ++i) {
            const int u = sum_upto64(count[i]);
            if (lane == 63) scr.sums[w][i] = u;
        }
        __syncthreads();
        int upto = 0;
#pragma unroll
        for (int i = 0; i < CLASSES; ++i) {
            begin[i] = upto;
#pragma unroll
            for (int j = 0; j < NW; ++j) upto += scr.sums[j][i];
        }
        __syncthreads();
    }
    for (int s0 = 0; s0 < n_seqs; s0 += NT) {
        if (s0) q = seq_of(s0 + tid);
        const int parts = parts_of(q), size = size_of(q, parts), c = class_of(size), items = q.tiles * parts;
        int mine[CLASSES + 1], upto[CLASSES + 1];
#pragma unroll
        for (int i = 0; i <= CLASSES; ++i) {
            mine[i] = i == CLASSES ? q.tiles : c == i ? items : 0;
            upto[i] = sum_upto64(mine[i]);
            if (lane == 63) scr.sums[w][i] = upto[i];
        }
        __syncthreads();
        int all = 0, at = 0, tile_at = 0;
#pragma unroll
        for (int i = 0; i <= CLASSES; ++i) {
            int here = (n_seqs > NT || i == CLASSES ? begin[i] : all) + upto[i] - mine[i];
#pragma unroll
            for (int j = 0; j < NW; ++j) {
                if (j < w) here += scr.sums[j][i];
                if (i < CLASSES) all += scr.sums[j][i];
                begin[i] += scr.sums[j][i];
            }
            if (i == CLASSES) tile_at = here;
            else if (c == i) at = here;
        }
        if (item >= at && item < at + items) {
            const int i = item - at, part = i / q.tiles, tile = i - part * q.tiles;      // (tiles of one part next to each other: they read the same rows)
            const int row0 = q.r0 + tile * a.tile_rows, rows = min(a.tile_rows, q.n - tile * a.tile_rows);
            scr.found[0] = s0 + tid;
            scr.found[1] = row0;
            scr.found[2] = rows;
            scr.found[3] = q.ctx;
            scr.found[4] = q.places - q.ctx;
            scr.found[5] = part;
            scr.found[6] = parts;
            scr.found[7] = size;
            if (hk == 0 && part == 0 && tile_at + tile < a.max_tiles) a.tiles[tile_at + tile] = {row0, rows, parts, at + tile, q.tiles, {}};
        }
        __syncthreads();
        if (scr.found[0] >= 0 && item != 0) break;       // (workgroup 0 counts all tiles)
    }
    if (item == 0 && hk == 0 && tid == 0) *a.n_tiles = min(begin[CLASSES], a.max_tiles);
    if (scr.found[0] < 0) return false;
    it.seq = scr.found[0], it.row0 = scr.found[1], it.rows = scr.found[2], it.ctx = scr.found[3], it.drafts = scr.found[4], it.parts = scr.found[6];
    const int places = it.ctx + it.drafts;
    it.lo = (int)min((long long)scr.found[5] * scr.found[7] * UNIT, (long long)places);
    it.hi = (int)min((long long)it.lo + (long long)scr.found[7] * UNIT, (long long)places);
    it.part_at = item;
    return true;
}

// Rows of no sequence: zeros.  The last workgroup of a K/V head.
template <int D, bool BF16, int NW>
__device__ __forceinline__ void clear_rows(const TreeArgs &a, int hk)
{
    const ListArgs &g = a.list;
    const int begin = g.n_seqs ? min(max(a.offsets[0], 0), g.T) : 0, end = g.n_seqs ? min(max(a.offsets[g.n_seqs], begin), g.T) : 0;
    const int chunks = (D << g.lg_g) * (BF16 ? 2 : 4) / 16;
    const size_t width = (size_t)g.Hq * D * (BF16 ? 2 : 4);
    auto clear = [&](int t0, int t1) {
        for (long long i = threadIdx.x; i < (long long)(t1 - t0) * chunks; i += 64 * NW)
            *(u32x4 *)((char *)g.out + (t0 + i / chunks) * width + ((size_t)hk * chunks + i % chunks) * 16) = (u32x4){0u, 0u, 0u, 0u};
    };
    clear(0, begin);
    clear(end, g.T);
}

// C columns: C >> lg_g rows of a sequence.
template <int D, int C, bool BF16>
__global__ __launch_bounds__(256) void tree_vector_kernel(TreeArgs a)
{
    __shared__ VectorScratch<C, D> scr;
    __shared__ TreeScratch find;
    __shared__ uint32_t bits[C][2 * ALORA_MAX_TREE_WORDS];
    const ListArgs &g = a.list;
    const int hk = (int)blockIdx.x % g.Hkv, item = (int)blockIdx.x / g.Hkv, tid = threadIdx.x;
    if (item == (int)(gridDim.x / g.Hkv) - 1) return clear_rows<D, BF16, 4>(a, hk);
    TreeItem it;
    if (!find_item<4>(a, item, hk, find, it)) return;
    const int G = 1 << g.lg_g;
    if (tid < 2 * a.words * it.rows) bits[tid / (2 * a.words)][tid % (2 * a.words)] = a.mask[(size_t)it.row0 * 2 * a.words + tid];
    __syncthreads();
    const int32_t *bt = g.bt + (size_t)it.seq * g.max_blocks;
    const auto column_at = [&](int c) { return (((long long)it.row0 + (c >> g.lg_g)) * g.Hq + hk * G + (c & (G - 1))) * D; };
    read_list_vector<D, C, BF16>(
        g, hk, scr, it.lo, it.hi, it.ctx,
        [&](int v) { return slot_at(g, bt, v / g.bs, v % g.bs); },
        [&](int c, int v) { return v < it.ctx || (bits[c >> g.lg_g][(v - it.ctx) >> 5] >> ((v - it.ctx) & 31) & 1u); },
        [&](int c) { return c >> g.lg_g < it.rows ? column_at(c) : -1ll; },
        [&](int c, int d, float M, float L, float o) {
            if (c >> g.lg_g >= it.rows) return;
            if (it.parts > 1) {
                const size_t at = ((size_t)it.part_at * g.Hkv + hk) * C + c;
                if (d == 0) *(f32x2 *)(g.ml + 2 * at) = (f32x2){M, L};
                g.o[at * D + d] = o;
                return;
            }
            const float y = L == 0.f ? 0.f : o / L;
            if (BF16) ((bf16_t *)g.out)[column_at(c) + d] = (bf16_t)f32_to_bf16_bits(y);
            else ((float *)g.out)[column_at(c) + d] = y;
        });
}

// 32 NW columns: 32 NW >> lg_g rows of a sequence.
template <int D, int NW, bool WHOLE, bool ONCE>
__global__ __launch_bounds__(64 * NW, 2) void tree_matrix_kernel(TreeArgs a)
{
    __shared__ MatrixTiles<D, NW, 32, 512 / D, 2, 2048> lds;      // 64 KiB of tiles: two workgroups share a CU's LDS
    __shared__ TreeScratch find;
    const ListArgs &g = a.list;
    const int hk = (int)blockIdx.x % g.Hkv, item = (int)blockIdx.x / g.Hkv;
    if (item == (int)(gridDim.x / g.Hkv) - 1) return clear_rows<D, true, NW>(a, hk);
    TreeItem it;
    if (!find_item<NW>(a, item, hk, find, it)) return;
    const int32_t *bt = g.bt + (size_t)it.seq * g.max_blocks;
    const int col = 32 * ((int)threadIdx.x >> 6) + ((int)threadIdx.x & 31), columns = it.rows << g.lg_g, row = it.row0 + (min(col, columns - 1) >> g.lg_g);
    const uint32_t *bits = a.mask + (size_t)row * 2 * a.words;
    const size_t at = ((size_t)row * g.Hq + ((size_t)hk << g.lg_g) + (col & ((1 << g.lg_g) - 1))) * D;
    read_list_matrix<WHOLE, ONCE>(
        g, hk, lds, it.lo, it.hi, it.ctx, columns,
        [&](int v) { return slot_at(g, bt, v / g.bs, v % g.bs); },
        [&](int place) {               // the row's bits of drafts place - ctx .. + 31; what lies in front of them is seen
            const int from = place - it.ctx, i = from >> 5, s = from & 31;
            const uint32_t x = i < 0 ? 0xffffffffu : i < 2 * a.words ? bits[i] : 0u, y = i + 1 < 2 * a.words ? bits[i + 1] : 0u;
            return s ? x >> s | y << (32 - s) : x;
        },
        at, at, it.parts > 1 ? (long long)it.part_at * g.Hkv + hk : -1ll, 32 * NW);
}

// One wavefront per column of a tile that has parts.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, int columns)
{
    const ListArgs &g = a.list;
    const int c = (int)blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hk = (int)blockIdx.x % g.Hkv, tile = (int)blockIdx.x / g.Hkv;
    if (tile >= *a.n_tiles) return;
    const TreeTile t = a.tiles[tile];
    if (t.parts <= 1 || c >> g.lg_g >= t.rows || (long long)t.first + (long long)(t.parts - 1) * t.step >= a.max_items) return;
    combine_parts<D, BF16>(g, (size_t)t.first * g.Hkv + hk, (size_t)t.step * g.Hkv, t.parts, columns, c,
                           ((size_t)(t.row0 + (c >> g.lg_g)) * g.Hq + ((size_t)hk << g.lg_g) + (c & ((1 << g.lg_g) - 1))) * D);
}

// ---- host ---------------------------------------------------------------------------------------
// How a call is cut: columns of a tile, the most tiles and items (tile, part) of a K/V head there can be, and where the workspace's arrays lie.
constexpr int WAVES = 4;
struct TreePlan {
    bool matrix;                // instructions; else vector arithmetic
    int columns, tile_rows, places;
    long long tiles, items;
    size_t tiles_at, ml_at, o_at, bytes;
};
static TreePlan plan_tree(const alora_attn_dims *d)
{
    TreePlan p;
    const int G = d->n_q_heads / d->n_kv_heads;
    p.matrix = d->dtype == ALORA_BF16;
    p.columns = p.matrix ? 32 * WAVES : 8;
    p.tile_rows = p.columns / G;
    p.places = std::max(1, 512 / d->n_kv_heads);
    p.tiles = d->n_tokens / p.tile_rows + std::min(d->n_seqs, d->n_tokens);      // (a sequence's last tile may not be full)
    p.items = p.tiles + p.places * 3 / 2 + 1;                                    // sum of ceil(units / per) over tiles, per >= all units / (1.5 places)
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    p.tiles_at = 256;
    p.ml_at = p.tiles_at + up((size_t)p.tiles * sizeof(TreeTile));
    p.o_at = p.ml_at + up((size_t)p.items * d->n_kv_heads * p.columns * 8);
    p.bytes = p.o_at + (size_t)p.items * d->n_kv_heads * p.columns * d->head_dim * 4;
    return p;
}

static int check_tree(const alora_attn_dims *d, int words)
{
    const int st = check_attention(d);
    if (st) return st;
    if (words < 1 || words > ALORA_MAX_TREE_WORDS || d->n_seqs > 1 << 20) return ALORA_ESHAPE;
    if (plan_tree(d).items * d->n_kv_heads > 0x3fffffffll) return ALORA_ESHAPE;
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
    if (!q || !k_cache || !v_cache || !block_tables || !row_offsets || !context_lens || !tree_mask || !out) return ALORA_EINVAL;
    if (((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)out) & 15 || (uintptr_t)tree_mask & 7) return ALORA_EINVAL;
    if (((uintptr_t)block_tables | (uintptr_t)row_offsets | (uintptr_t)context_lens) & 3) return ALORA_EINVAL;
    TreeArgs a;
    a.list = list_args(dims, q, k_cache, v_cache, block_tables, out);
    a.list.ml = (float *)((char *)workspace + p.ml_at);
    a.list.o = (float *)((char *)workspace + p.o_at);
    a.offsets = row_offsets; a.context = context_lens;
    a.mask = (const uint32_t *)tree_mask; a.words = mask_words;
    a.tile_rows = p.tile_rows; a.places = p.places;
    a.max_tiles = (int)p.tiles; a.max_items = (int)p.items;
    a.n_tiles = (int *)workspace;
    a.tiles = (TreeTile *)((char *)workspace + p.tiles_at);
    const bool bf16 = dims->dtype == ALORA_BF16;
    const dim3 grid((unsigned)((p.items + 1) * dims->n_kv_heads)), merge((unsigned)(p.tiles * dims->n_kv_heads), (unsigned)p.columns / 4);
    const auto go = [&](auto kernel, auto combine) {
        launch_kernel(kernel, grid, dim3(64 * WAVES), 0, (hipStream_t)hip_stream, a);
        launch_kernel(combine, merge, dim3(256), 0, (hipStream_t)hip_stream, a, p.columns);
    };
    // Weights whole where a sequence brings one wavefront's columns on average: then the call waits for memory.  Non-temporal copies where it brings one tile, so
    // that its context is read once, and the memory-side cache would not keep K and V.  us, ordinary | non-temporal | with whole weights, 32/8 heads, 8192
    // positions: 64 x 1 rows 376 | | 341, 64 x 8 379 | | 344, 2000 positions: 300 x 4 480 | | 452; 64/8 heads, 64 rows at 64000, four tiles 181 | | 245.
    const long long columns = (long long)dims->n_tokens * (dims->n_q_heads / dims->n_kv_heads);
    const bool whole = columns <= 32ll * dims->n_seqs;
    const bool once = columns <= 32ll * WAVES * dims->n_seqs && outgrows_cache(dims->n_slots, dims->n_kv_heads, dims->head_dim, true);
    const auto choose = [&](auto head_dim) {
        constexpr int D = decltype(head_dim)::value;
        if (!bf16) go(tree_vector_kernel<D, 8, false>, tree_merge_kernel<D, false>);
        else if (whole) once ? go(tree_matrix_kernel<D, WAVES, true, true>, tree_merge_kernel<D, true>) : go(tree_matrix_kernel<D, WAVES, true, false>, tree_merge_kernel<D, true>);
        else once ? go(tree_matrix_kernel<D, WAVES, false, true>, tree_merge_kernel<D, true>) : go(tree_matrix_kernel<D, WAVES, false, false>, tree_merge_kernel<D, true>);
    };
    if (dims->head_dim == 128) choose(std::integral_constant<int, 128>{});
    else choose(std::integral_constant<int, 64>{});
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

}  // extern "C"
