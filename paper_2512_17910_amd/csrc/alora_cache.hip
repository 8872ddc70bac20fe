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
struct CacheTable {
    char *p[2 * LAYERS_AT_ONCE];    // K and V of layer 0, K and V of layer 1, ...
};
template <int PAIRS>
struct PairList {
    int32_t src[PAIRS], dst[PAIRS];
};
constexpr int PAIRS_FEW = 16, PAIRS_MANY = 352;
static_assert(sizeof(CacheTable) + sizeof(PairList<PAIRS_MANY>) + 16 <= 4096, "kernel arguments");

// One workgroup per piece of 4 KiB * K of a block, cache and pair.
template <int PAIRS, int K>
__global__ __launch_bounds__(256) void copy_blocks_kernel(CacheTable caches, PairList<PAIRS> pairs, long long block_bytes)
{
    char *cache = caches.p[blockIdx.y];
    const int src = pairs.src[blockIdx.z], dst = pairs.dst[blockIdx.z];
    const long long piece = (long long)blockIdx.x * (K * 4096);
    const int left = (int)min(block_bytes - piece, (long long)K * 4096), o = threadIdx.x * 16;
    const char *from = cache + src * block_bytes + piece;    // (not read where src is -1)
    char *to = cache + dst * block_bytes + piece;
    u32x4 x[K];
    if (left == K * 4096) {
#pragma unroll
        for (int i = 0; i < K; ++i) x[i] = u32x4{0u, 0u, 0u, 0u};
        if (src >= 0) {
#pragma unroll
            for (int i = 0; i < K; ++i) x[i] = *(const u32x4 *)(from + o + i * 4096);
        }
#pragma unroll
        for (int i = 0; i < K; ++i) *(u32x4 *)(to + o + i * 4096) = x[i];
        return;
    }
    for (int i = o; i < left; i += 4096) *(u32x4 *)(to + i) = src >= 0 ? *(const u32x4 *)(from + i) : u32x4{0u, 0u, 0u, 0u};
}

struct MoveArgs {
    CacheTable caches;
    const int64_t *src, *dst;
    const int32_t *shift;       // or null
    const float *cos, *sin;
    HeadShape s;
    int hkv, n_pos, uk;         // uk: units of 64 >> gshift heads
    int layers, per_group;      // per_group: layers of a workgroup
    int n_rows;
    long long n_slots, row_bytes;
};

constexpr int MOVE_WAVES = 8;
constexpr int MOVE_LAYERS = 4;   // layers whose loads are requested together

// One workgroup per row and group of layers.  A wavefront takes a unit of key heads or 2 KiB of values through the layers; its
// angles are the same in all of them.
template <bool BF16, int V, bool INTERLEAVED>
__global__ __launch_bounds__(64 * MOVE_WAVES) void move_rows_kernel(MoveArgs g)
{
    typedef Chunk<BF16, V> C;
    constexpr int E = BF16 ? 2 : 4, L = MOVE_LAYERS;
    const long long row = (long long)blockIdx.z * ROWS_AT_ONCE + blockIdx.x;
    if (row >= g.n_rows) return;
    const long long src = g.src[row], dst = g.dst[row];
    if (src < 0 || src >= g.n_slots || dst < 0 || dst >= g.n_slots) return;
    const int shift = g.shift ? g.shift[row] : 0;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    const int l0 = blockIdx.y * g.per_group, l1 = min(l0 + g.per_group, g.layers);
    const int pieces = (int)((g.row_bytes + 2047) / 2048), k_units = shift ? g.uk : pieces;
    const LanePlace p = lane_place<V, INTERLEAVED>(g.s, lane & ((1 << g.s.gshift) - 1));
    float c[V], s[V];
    if (shift && wave < k_units) {
        const uint32_t far = shift < 0 ? 0u - (uint32_t)shift : (uint32_t)shift;
        load_angles<V, INTERLEAVED>(g.cos, g.sin, (size_t)min(far, (uint32_t)g.n_pos - 1u) * g.s.half, p, c, s);
        if (shift < 0) {
#pragma unroll
            for (int e = 0; e < V; ++e) s[e] = -s[e];
        }
    }
    for (int u = wave; u < k_units + pieces; u += waves) {
        if (shift && u < k_units) {
            const int head = u * (64 >> g.s.gshift) + (lane >> g.s.gshift);
            const bool on = head < g.hkv;
            const long long offset = (long long)head * (g.s.d * E);
            for (int l = l0; l < l1; l += L) {
                C a[L], b[L];
#pragma unroll
                for (int i = 0; i < L; ++i) {
                    a[i].zero();
                    b[i].zero();
                    if (l + i < l1) {
                        const char *from = g.caches.p[2 * (l + i)] + src * g.row_bytes + offset;
                        if (on && p.has_a) a[i].load(from + p.a * E);
                        if (on && p.has_b) b[i].load(from + p.b * E);
                    }
                }
#pragma unroll
                for (int i = 0; i < L; ++i) {
                    float x[V], y[V];
                    a[i].widen(x);
                    b[i].widen(y);
                    turn<V, INTERLEAVED, false>(x, y, c, s, p);
                    a[i].narrow(x);
                    b[i].narrow(y);
                    if (l + i < l1) {
                        char *to = g.caches.p[2 * (l + i)] + dst * g.row_bytes + offset;
                        if (on && p.has_a) a[i].store(to + p.a * E);
                        if (on && p.has_b) b[i].store(to + p.b * E);
                    }
                }
            }
            continue;
        }
        const int side = u < k_units ? 0 : 1;
        const long long o = (long long)(side ? u - k_units : u) * 2048 + lane * 16;
        for (int l = l0; l < l1; l += L) {
            u32x4 x[L], y[L];
#pragma unroll
            for (int i = 0; i < L; ++i) {
                if (l + i >= l1) break;
                const char *from = g.caches.p[2 * (l + i) + side] + src * g.row_bytes + o;
                if (o < g.row_bytes) x[i] = *(const u32x4 *)from;
                if (o + 1024 < g.row_bytes) y[i] = *(const u32x4 *)(from + 1024);
            }
#pragma unroll
            for (int i = 0; i < L; ++i) {
                if (l + i >= l1) break;
                char *to = g.caches.p[2 * (l + i) + side] + dst * g.row_bytes + o;
                if (o < g.row_bytes) *(u32x4 *)to = x[i];
                if (o + 1024 < g.row_bytes) *(u32x4 *)(to + 1024) = y[i];
            }
        }
    }
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

static CacheTable table_of(const alora_cache_dims *d, int first, int n)
{
    CacheTable t;
    for (int l = 0; l < LAYERS_AT_ONCE; ++l) {
        t.p[2 * l] = (char *)(l < n ? d->k_caches[first + l] : nullptr);
        t.p[2 * l + 1] = (char *)(l < n ? d->v_caches[first + l] : nullptr);
    }
    return t;
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

template <int PAIRS>
static void launch_copies(const CacheTable &caches, int n_caches, const int32_t *src, const int32_t *dst, int n, long long block_bytes, hipStream_t st)
{
    for (int i = 0; i < n; i += PAIRS) {
        const int m = std::min(PAIRS, n - i);
        PairList<PAIRS> list;
        std::copy(src + i, src + i + m, list.src);
        std::copy(dst + i, dst + i + m, list.dst);
        // pieces of 32 KiB where that gives the chip two workgroups for every compute unit, else of 4
        const long long large = (block_bytes + 32767) / 32768;
        if (large * n_caches * m >= 512)
            launch_kernel(copy_blocks_kernel<PAIRS, 8>, dim3((unsigned)large, n_caches, m), dim3(256), 0, st, caches, list, block_bytes);
        else
            launch_kernel(copy_blocks_kernel<PAIRS, 1>, dim3((unsigned)((block_bytes + 4095) / 4096), n_caches, m), dim3(256), 0, st, caches, list, block_bytes);
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
    for (int l = 0; l < dims->n_layers; l += LAYERS_AT_ONCE) {
        const int layers = std::min(LAYERS_AT_ONCE, dims->n_layers - l);
        const CacheTable caches = table_of(dims, l, layers);
        if (n <= PAIRS_FEW) launch_copies<PAIRS_FEW>(caches, 2 * layers, src, dst, n, block_bytes, (hipStream_t)hip_stream);
        else launch_copies<PAIRS_MANY>(caches, 2 * layers, src, dst, n, block_bytes, (hipStream_t)hip_stream);
    }
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
    if ((shift != nullptr) != (rotary_dim > 0) || (cos != nullptr) != (rotary_dim > 0) || (sin != nullptr) != (rotary_dim > 0)) return ALORA_EINVAL;
    if (rotary_dim && rope_positions < 1) return ALORA_EINVAL;
    if (n_rows == 0 || dims->n_layers == 0) return ALORA_OK;
    if (!src || !dst) return ALORA_EINVAL;
    if ((((uintptr_t)src | (uintptr_t)dst) & 7) || ((uintptr_t)shift & 3) || (((uintptr_t)cos | (uintptr_t)sin) & 15)) return ALORA_EINVAL;
    st = check_pointers(dims);
    if (st) return st;
    const bool bf16 = dims->dtype == ALORA_BF16;
    const int V = head_chunk(bf16, rotary_dim, interleaved);
    MoveArgs g;
    g.n_rows = n_rows;
    g.src = src; g.dst = dst; g.shift = shift; g.cos = cos; g.sin = sin;
    g.s = head_shape(dims->head_dim, rotary_dim, interleaved, V);
    g.hkv = dims->n_kv_heads; g.n_pos = rope_positions;
    const int per = 64 >> g.s.gshift;
    g.uk = (g.hkv + per - 1) / per;
    g.n_slots = dims->n_slots;
    g.row_bytes = row_bytes_of(dims);
    const long long pieces = (g.row_bytes + 2047) / 2048, units = pieces + (shift ? std::max<long long>(g.uk, pieces) : pieces);
    const int waves = (int)std::min<long long>(MOVE_WAVES, units);
    for (int l = 0; l < dims->n_layers; l += LAYERS_AT_ONCE) {
        g.layers = std::min(LAYERS_AT_ONCE, dims->n_layers - l);
        g.caches = table_of(dims, l, g.layers);
        // all layers of a row on one workgroup where the rows alone fill the chip, else MOVE_LAYERS or one
        g.per_group = (long long)n_rows * waves >= 8192 ? g.layers : (long long)n_rows * waves * g.layers >= 8192 ? MOVE_LAYERS : 1;
        const dim3 grid(std::min(n_rows, ROWS_AT_ONCE), (g.layers + g.per_group - 1) / g.per_group, (n_rows - 1) / ROWS_AT_ONCE + 1), block(64 * waves);
        const auto go = [&](auto kernel) { launch_kernel(kernel, grid, block, 0, (hipStream_t)hip_stream, g); };
        if (bf16 && V == 8) interleaved ? go(move_rows_kernel<true, 8, true>) : go(move_rows_kernel<true, 8, false>);
        else if (bf16 && V == 4) go(move_rows_kernel<true, 4, false>);
        else if (bf16) interleaved ? go(move_rows_kernel<true, 2, true>) : go(move_rows_kernel<true, 2, false>);
        else if (V == 4) interleaved ? go(move_rows_kernel<false, 4, true>) : go(move_rows_kernel<false, 4, false>);
        else interleaved ? go(move_rows_kernel<false, 2, true>) : go(move_rows_kernel<false, 2, false>);
    }
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
