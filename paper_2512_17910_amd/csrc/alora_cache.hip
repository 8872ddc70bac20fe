// Copies of cache blocks and moves of token rows over all layers (include/alora_cache.h).
#include <algorithm>
#include <new>
#include <vector>
#include "alora_cache.h"
#include "alora_heads_core.h"

namespace alora {

// Addresses and block pairs go to the kernel with its arguments (at most 4 KiB of them): a copy needs no memory of its own on the device, and
// the lists may be read before the call returns.
constexpr int LAYERS_AT_ONCE = 64;
template <int LAYERS>
struct CacheTable {
    char *p[2 * LAYERS];    // K and V of layer 0, K and V of layer 1, ...
};
template <int PAIRS>
struct PairList {
    int32_t src[PAIRS], dst[PAIRS];
};
constexpr int PAIRS_FEW = 16, PAIRS_MANY = 352;
static_assert(sizeof(CacheTable<LAYERS_AT_ONCE>) + sizeof(PairList<PAIRS_MANY>) + 16 <= 4096, "kernel arguments");

// One workgroup per piece of 4 KiB of a block, pair and cache; all pairs of a cache before the next cache.  Bound by memory: each byte is
// read and written once, past the caches, since nothing reads it soon.  1000 blocks of 32 KiB in 16 caches, us: 200 (5.2 TB/s, what a
// large copy reaches), with ordinary loads and stores 4 to 8 % more, with the caches of a pair behind each other 3 % more; 724 blocks of 8 KiB in 16
// caches 39.5.  Pieces of 8, 16, 32 KiB: 204, 205, 204 and 41.5, 45.3, 45.3.  One block in 64 caches takes 2.6 us: a launch.
template <int LAYERS, int PAIRS>
__global__ __launch_bounds__(256) void copy_blocks_kernel(CacheTable<LAYERS> caches, PairList<PAIRS> pairs, long long block_bytes)
{
    char *cache = caches.p[blockIdx.z];
    const int src = pairs.src[blockIdx.y], dst = pairs.dst[blockIdx.y];
    const long long at = (long long)blockIdx.x * 4096 + threadIdx.x * 16;
    if (at >= block_bytes) return;
    u32x4 x = {0u, 0u, 0u, 0u};
    if (src >= 0) x = __builtin_nontemporal_load((const u32x4 *)(cache + src * block_bytes + at));
    __builtin_nontemporal_store(x, (u32x4 *)(cache + dst * block_bytes + at));
}

// How rows lie on wavefronts: `rows` of them on one where they leave room, else one on `units`.  Bound by memory; what costs next is the number of
// wavefronts, each with a chain of loads (indexes, shift; angles and rows).  9001 rows over 16 layers, us: 8 heads of 128 219 (5.4 TB/s), in
// wavefronts that went through four layers each 245; one head of 64 19 (a row to a workgroup: 44, a row and layer: 93).
struct RowSplit {
    int rows, units;
};

struct MoveArgs {
    const int64_t *src, *dst;
    const int32_t *shift;       // or null
    const float *cos, *sin;
    HeadShape s;
    RowSplit k, v;              // of keys that are turned; of rows that are copied, in 16-byte pieces
    int heads, pieces, n_rows, n_pos;
    long long n_slots, row_bytes;
};

struct Move {
    long long src, dst;
    bool on;
};
__device__ __forceinline__ Move move_of(const MoveArgs &g, int row)
{
    Move m = {g.src[row], g.dst[row], false};
    m.on = m.src >= 0 && m.src < g.n_slots && m.dst >= 0 && m.dst < g.n_slots;
    return m;
}

constexpr int MOVE_WAVES = 4;

// A wavefront's share of a layer's K cache, keys turned on the way.
template <bool BF16, int V, bool INTERLEAVED>
__device__ __forceinline__ void move_keys(const MoveArgs &g, char *cache, int item, int lane)
{
    typedef Chunk<BF16, V> C;
    constexpr int E = BF16 ? 2 : 4;
    const LanePlace p = lane_place<V, INTERLEAVED>(g.s, lane & ((1 << g.s.gshift) - 1));
    const int h = lane >> g.s.gshift;
    const int group = g.k.units == 1 ? item : item / g.k.units;
    if (group >= (g.n_rows + g.k.rows - 1) / g.k.rows) return;
    int row = group, head = (item - group * g.k.units) * (64 >> g.s.gshift) + h;
    Move m;
    int shift;
    bool on = head < g.heads;
    if (g.k.rows == 1) {       // (one row: scalar loads)
        m = move_of(g, row);
        shift = g.shift[row];
    } else {
        const int sub = h / g.heads;
        head = h - sub * g.heads;
        row = group * g.k.rows + sub;
        on = sub < g.k.rows && row < g.n_rows;
        row = min(row, g.n_rows - 1);
        m = move_of(g, row);
        shift = g.shift[row];
    }
    on &= m.on;
    if (!on) return;
    const char *from = cache + m.src * g.row_bytes + head * (g.s.d * E);
    char *to = cache + m.dst * g.row_bytes + head * (g.s.d * E);
    C a, b;
    a.zero();
    b.zero();
    if (p.has_a) a.load(from + p.a * E);
    if (p.has_b) b.load(from + p.b * E);
    if (shift) {      // (keys that keep their position are copied bit for bit)
        const uint32_t far = shift < 0 ? 0u - (uint32_t)shift : (uint32_t)shift;
        float c[V], s[V], x[V], y[V];
        load_angles<V, INTERLEAVED>(g.cos, g.sin, (size_t)min(far, (uint32_t)g.n_pos - 1u) * g.s.half, p, c, s);
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] = shift < 0 ? -s[e] : s[e];
        a.widen(x);
        b.widen(y);
        turn<V, INTERLEAVED, false>(x, y, c, s, p);
        a.narrow(x);
        b.narrow(y);
    }
    if (p.has_a) a.store(to + p.a * E);
    if (p.has_b) b.store(to + p.b * E);
}

// A wavefront's share of a cache whose rows are copied as they are: 2 KiB, past the caches.  (Turned keys are loaded and stored the ordinary way: chunks of
// their layout cover lines in two requests.)
__device__ __forceinline__ void move_copies(const MoveArgs &g, char *cache, int item, int lane)
{
    const int group = g.v.units == 1 ? item : item / g.v.units;
    if (group >= (g.n_rows + g.v.rows - 1) / g.v.rows) return;
    u32x4 x[2];
    char *to[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        to[i] = nullptr;
        int piece = (item - group * g.v.units) * 128 + 64 * i + lane;
        Move m;
        bool on = piece < g.pieces;
        if (g.v.rows == 1) {
            m = move_of(g, group);
        } else {
            const int sub = piece / g.pieces, row = group * g.v.rows + sub;
            piece -= sub * g.pieces;
            on = sub < g.v.rows && row < g.n_rows;
            m = move_of(g, min(row, g.n_rows - 1));
        }
        if (on && m.on) {
            x[i] = __builtin_nontemporal_load((const u32x4 *)(cache + m.src * g.row_bytes + piece * 16));
            to[i] = cache + m.dst * g.row_bytes + piece * 16;
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (to[i]) __builtin_nontemporal_store(x[i], (u32x4 *)to[i]);
}

// One wavefront per item of a layer's K or V cache; gridDim.y counts the caches.
template <int LAYERS, bool BF16, int V, bool INTERLEAVED>
__global__ __launch_bounds__(64 * MOVE_WAVES) void move_rows_kernel(CacheTable<LAYERS> caches, MoveArgs g)
{
    const int item = blockIdx.x * MOVE_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    char *cache = caches.p[blockIdx.y];
    if (g.shift && !(blockIdx.y & 1)) move_keys<BF16, V, INTERLEAVED>(g, cache, item, lane);
    else move_copies(g, cache, item, lane);
}

// ---- host ---------------------------------------------------------------------------------------
static int check_cache(const alora_cache_dims *d)
{
    if (!d) return ALORA_EINVAL;
    if (d->dtype != ALORA_F32 && d->dtype != ALORA_BF16) return ALORA_EINVAL;
    if (d->n_layers < 0 || d->n_kv_heads < 1 || d->head_dim < 1 || d->block_size < 1 || d->n_slots < 0) return ALORA_EINVAL;
    if (d->head_dim > 256 || d->head_dim % (d->dtype == ALORA_BF16 ? 8 : 4) || d->n_kv_heads > 0x3fffffff / d->head_dim) return ALORA_ESHAPE;
    if (d->n_slots % d->block_size || d->n_slots / d->block_size > 0x7fffffffll || d->n_layers > 4096) return ALORA_ESHAPE;
    const long long row = (long long)d->n_kv_heads * d->head_dim * (d->dtype == ALORA_BF16 ? 2 : 4);
    if (d->n_slots > (1ll << 52) / row || row * d->block_size > 0x7fffffffll) return ALORA_ESHAPE;
    return ALORA_OK;
}

static int check_pointers(const alora_cache_dims *d)
{
    if (!d->k_caches || !d->v_caches) return ALORA_EINVAL;
    for (int l = 0; l < d->n_layers; ++l)
        if (!d->k_caches[l] || !d->v_caches[l] || (((uintptr_t)d->k_caches[l] | (uintptr_t)d->v_caches[l]) & 15)) return ALORA_EINVAL;
    return ALORA_OK;
}

// f(table, number of its layers) for every LAYERS_AT_ONCE layers, with a table of 8, 32 or 64: arguments are written across the bus, and cost
// 0.3 us for every 512 bytes (one block in 64 caches, the pass: 5.6 us with a table of 64 layers, 5.3 with one of 32).
template <typename F>
static void for_layers(const alora_cache_dims *d, F f)
{
    const auto with = [&](auto table, int first, int n) {
        for (int l = 0; l < n; ++l) {
            table.p[2 * l] = (char *)d->k_caches[first + l];
            table.p[2 * l + 1] = (char *)d->v_caches[first + l];
        }
        f(table, n);
    };
    for (int first = 0; first < d->n_layers; first += LAYERS_AT_ONCE) {
        const int n = std::min(LAYERS_AT_ONCE, d->n_layers - first);
        if (n <= 8) with(CacheTable<8>(), first, n);
        else if (n <= 32) with(CacheTable<32>(), first, n);
        else with(CacheTable<LAYERS_AT_ONCE>(), first, n);
    }
}

static long long row_bytes_of(const alora_cache_dims *d) { return (long long)d->n_kv_heads * d->head_dim * (d->dtype == ALORA_BF16 ? 2 : 4); }

// every destination once, and no block on both sides
static int check_pairs(const int32_t *src, const int32_t *dst, int n, long long blocks)
{
    for (int i = 0; i < n; ++i)
        if (src[i] < -1 || src[i] >= blocks || dst[i] < 0 || dst[i] >= blocks) return ALORA_EDATA;
    if (n <= PAIRS_FEW) {
        for (int i = 0; i < n; ++i)
            for (int j = 0; j < n; ++j)
                if (dst[i] == src[j] || (i != j && dst[i] == dst[j])) return ALORA_EDATA;
        return ALORA_OK;
    }
    try {
        // A short list of a large pool: sorting it takes less than clearing a bit for every block.  us sorted | with bits, words of bits per block of the
        // list 64, 128, 512: 64 blocks 0.8 | 0.3, 1.3, 5.5; 256 blocks 4.3 | 2.9, 5.8, 22; 1000 blocks 75 | 12, 23, 153 (one core of a host).
        if (blocks / 64 > 128ll * n) {
            std::vector<int32_t> sorted(dst, dst + n);
            std::sort(sorted.begin(), sorted.end());
            if (std::adjacent_find(sorted.begin(), sorted.end()) != sorted.end()) return ALORA_EDATA;
            for (int i = 0; i < n; ++i)
                if (src[i] >= 0 && std::binary_search(sorted.begin(), sorted.end(), src[i])) return ALORA_EDATA;
            return ALORA_OK;
        }
        std::vector<uint64_t> written((size_t)(blocks + 63) / 64, 0);
        for (int i = 0; i < n; ++i) {
            uint64_t &w = written[(size_t)dst[i] / 64];
            const uint64_t bit = 1ull << (dst[i] % 64);
            if (w & bit) return ALORA_EDATA;
            w |= bit;
        }
        for (int i = 0; i < n; ++i)
            if (src[i] >= 0 && (written[(size_t)src[i] / 64] >> (src[i] % 64) & 1)) return ALORA_EDATA;
    } catch (const std::bad_alloc &) {
        return ALORA_ENOMEM;
    }
    return ALORA_OK;
}

template <int PAIRS, int LAYERS>
static void launch_copies(const CacheTable<LAYERS> &caches, int n_caches, const int32_t *src, const int32_t *dst, int n, long long block_bytes, hipStream_t st)
{
    for (int i = 0; i < n; i += PAIRS) {
        const int m = std::min(PAIRS, n - i);
        PairList<PAIRS> list;
        std::copy(src + i, src + i + m, list.src);
        std::copy(dst + i, dst + i + m, list.dst);
        launch_kernel(copy_blocks_kernel<LAYERS, PAIRS>, dim3((unsigned)((block_bytes + 4095) / 4096), m, n_caches), dim3(256), 0, st, caches, list, block_bytes);
    }
}

}  // namespace alora

using namespace alora;

extern "C" {

int alora_cache_copy_blocks(const int32_t *src, const int32_t *dst, int32_t n, const alora_cache_dims *dims, void *hip_stream)
{
    int st = check_cache(dims);
    if (st) return st;
    if (n < 0 || (n && (!src || !dst))) return ALORA_EINVAL;
    if (n == 0 || dims->n_layers == 0) return ALORA_OK;
    st = check_pointers(dims);
    if (!st) st = check_pairs(src, dst, n, dims->n_slots / dims->block_size);
    if (st) return st;
    const long long block_bytes = row_bytes_of(dims) * dims->block_size;
    for_layers(dims, [&](const auto &caches, int layers) {
        if (n <= PAIRS_FEW) launch_copies<PAIRS_FEW>(caches, 2 * layers, src, dst, n, block_bytes, (hipStream_t)hip_stream);
        else launch_copies<PAIRS_MANY>(caches, 2 * layers, src, dst, n, block_bytes, (hipStream_t)hip_stream);
    });
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

int alora_cache_move_rows(const int64_t *src, const int64_t *dst, const int32_t *shift, int32_t n_rows, const float *cos, const float *sin,
                          int32_t rope_positions, int32_t rotary_dim, int32_t interleaved, const alora_cache_dims *dims, void *hip_stream)
{
    int st = check_cache(dims);
    if (st) return st;
    if (n_rows < 0 || rotary_dim < 0 || (interleaved | 1) != 1) return ALORA_EINVAL;
    if (rotary_dim % 4 || rotary_dim > dims->head_dim) return ALORA_ESHAPE;
    if (rotary_dim && rope_positions < 1) return ALORA_EINVAL;
    if ((long long)n_rows * dims->n_kv_heads > 1 << 25) return ALORA_ESHAPE;     // (a grid holds fewer than 2^32 threads)
    if (n_rows == 0 || dims->n_layers == 0) return ALORA_OK;
    if (!src || !dst) return ALORA_EINVAL;
    if ((shift != nullptr) != (rotary_dim > 0) || (cos != nullptr) != (rotary_dim > 0) || (sin != nullptr) != (rotary_dim > 0)) return ALORA_EINVAL;
    if ((((uintptr_t)src | (uintptr_t)dst) & 7) || ((uintptr_t)shift & 3) || (((uintptr_t)cos | (uintptr_t)sin) & 15)) return ALORA_EINVAL;
    st = check_pointers(dims);
    if (st) return st;
    const bool bf16 = dims->dtype == ALORA_BF16;
    const int V = head_chunk(bf16, dims->head_dim, rotary_dim, interleaved);
    MoveArgs g;
    g.src = src; g.dst = dst; g.shift = shift; g.cos = cos; g.sin = sin;
    g.heads = dims->n_kv_heads; g.n_rows = n_rows; g.n_pos = rope_positions;
    g.s = head_shape(dims->head_dim, rotary_dim, interleaved, V);
    g.n_slots = dims->n_slots;
    g.row_bytes = row_bytes_of(dims);
    g.pieces = (int)(g.row_bytes / 16);
    const auto split = [](int parts, int at_once) { return RowSplit{std::max(1, at_once / parts), (parts + at_once - 1) / at_once}; };
    g.k = split(g.heads, 64 >> g.s.gshift);
    g.v = split(g.pieces, 128);
    const auto items = [&](const RowSplit &x) { return ((long long)n_rows + x.rows - 1) / x.rows * x.units; };
    const long long groups = (std::max(items(g.v), shift ? items(g.k) : 0) + MOVE_WAVES - 1) / MOVE_WAVES;
    for_layers(dims, [&](const auto &caches, int layers) {
        constexpr int L = sizeof(caches) / (2 * sizeof(char *));
        const auto go = [&](auto kernel) { launch_kernel(kernel, dim3((unsigned)groups, 2 * layers), dim3(64 * MOVE_WAVES), 0, (hipStream_t)hip_stream, caches, g); };
        if (bf16 && V == 8) interleaved ? go(move_rows_kernel<L, true, 8, true>) : go(move_rows_kernel<L, true, 8, false>);
        else if (bf16 && V == 4) interleaved ? go(move_rows_kernel<L, true, 4, true>) : go(move_rows_kernel<L, true, 4, false>);
        else if (bf16) go(move_rows_kernel<L, true, 2, false>);
        else if (V == 4) interleaved ? go(move_rows_kernel<L, false, 4, true>) : go(move_rows_kernel<L, false, 4, false>);
        else go(move_rows_kernel<L, false, 2, false>);
    });
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

int alora_cache_move_rows_validate(const int64_t *src, const int64_t *dst, const int32_t *shift, int32_t n_rows, int32_t rope_positions,
                                   const alora_cache_dims *dims)
{
    const int st = check_cache(dims);
    if (st) return st;
    if (n_rows < 0) return ALORA_EINVAL;
    if (n_rows == 0) return ALORA_OK;
    if (!src || !dst) return ALORA_EINVAL;
    try {
        const size_t n = (size_t)n_rows;
        std::vector<int64_t> s(n), d(n);
        std::vector<int32_t> sh(shift ? n : 0);
        hipError_t e = hipMemcpy(s.data(), src, 8 * n, hipMemcpyDeviceToHost);
        if (!e) e = hipMemcpy(d.data(), dst, 8 * n, hipMemcpyDeviceToHost);
        if (!e && shift) e = hipMemcpy(sh.data(), shift, 4 * n, hipMemcpyDeviceToHost);
        if (e) { note_hip_error((int)e); return ALORA_EHIP; }
        for (size_t i = 0; i < n; ++i)
            if (s[i] < 0 || s[i] >= dims->n_slots || d[i] < 0 || d[i] >= dims->n_slots) return ALORA_EDATA;
        for (int32_t x : sh)
            if (x <= -rope_positions || x >= rope_positions) return ALORA_EDATA;
        std::vector<size_t> order(n);
        for (size_t i = 0; i < n; ++i) order[i] = i;
        std::sort(order.begin(), order.end(), [&](size_t a, size_t b) { return d[a] < d[b]; });
        for (size_t i = 1; i < n; ++i)
            if (d[order[i]] == d[order[i - 1]]) return ALORA_EDATA;
        for (size_t i = 0; i < n; ++i) {      // the row that writes slot s[i], if any, has to be this one
            const auto at = std::lower_bound(order.begin(), order.end(), s[i], [&](size_t a, int64_t v) { return d[a] < v; });
            if (at != order.end() && d[*at] == s[i] && *at != i) return ALORA_EDATA;
        }
        return ALORA_OK;
    } catch (const std::bad_alloc &) {
        return ALORA_ENOMEM;
    }
}

}  // extern "C"
