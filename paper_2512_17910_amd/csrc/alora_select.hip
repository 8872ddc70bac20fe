// Long contexts read in part (include/alora_select.h): bounds of the blocks' keys, the blocks to be read, attention over those.
#include <algorithm>
#include "alora_select.h"
#include "alora_listed.h"

namespace alora {

// ---- bounds ---------------------------------------------------------------------------------------
struct BoundsArgs {
    const void *kc;
    const int64_t *slot;
    int8_t *bounds;
    float *scales;
    int n_rows, Hkv, bs, units;      // units: wavefronts a cache row takes (64 pieces of 8 elements each)
    long long n_slots;
};

constexpr float TINY = 0x1p-100f;    // bounds and queries below it count as zero
constexpr float LARGEST = 3.402823466e38f;

// A lane keeps 8 components of a head through all rows of the block: nothing is exchanged before the largest component of a head is wanted.  A
// workgroup looks over ROWS rows of the call for the last ones of their blocks; its wavefronts take those in turn, `units` each.
template <int D, bool BF16, int ROWS>
__global__ __launch_bounds__(256) void block_bounds_kernel(BoundsArgs a)
{
    constexpr int LPH = D / 8;       // lanes per head
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = (int)blockIdx.x * ROWS, row = row0 + lane;
    auto block_of = [&](long long slot) { return slot >= 0 && slot < a.n_slots ? (int)slot / a.bs : -1; };
    const long long slot = row < a.n_rows ? a.slot[row] : -1;
    const int block = block_of(slot), off = block >= 0 ? (int)slot - block * a.bs : 0;
    // the block of the next row that has one: mostly the next lane's
    const unsigned long long have = __builtin_amdgcn_ballot_w64(block >= 0), later = lane < 63 ? have >> (lane + 1) : 0ull;
    int next = __shfl(block, later ? lane + 1 + (int)__builtin_ctzll(later) : 63);
    if (!later) next = -1;
    if (have && (int)(63 - __builtin_clzll(have)) < ROWS) {      // (the last of these may be followed from further on)
        for (long long j = row0 + 64ll; j < a.n_rows; j += 64) {
            const int far = block_of(j + lane < a.n_rows ? a.slot[j + lane] : -1);
            const unsigned long long any = __builtin_amdgcn_ballot_w64(far >= 0);
            if (!any) continue;
            const int found = __builtin_amdgcn_readlane(far, (int)__builtin_ctzll(any));
            if (!later) next = found;
            break;
        }
    }
    const bool last = lane < ROWS && block >= 0 && next != block;
    unsigned long long todo = __builtin_amdgcn_ballot_w64(last);
    const size_t width = (size_t)a.Hkv * D;
    const int n = (int)__builtin_popcountll(todo) * a.units;
    int at = 0;                      // leading rows already taken from todo
    for (int i = w; i < n; i += 4) {
        const int which = i / a.units, piece = (i - which * a.units) * 64 + lane;
        for (; at < which; ++at) todo &= todo - 1;
        const int from = (int)__builtin_ctzll(todo);
        const int b = __builtin_amdgcn_readlane(block, from), rows = __builtin_amdgcn_readlane(off, from) + 1;
        const bool on = piece * 8 < (int)width;
        float lo[8], hi[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) lo[e] = __builtin_inff(), hi[e] = -__builtin_inff();
        bool fine = true;
        if (on) {
            const size_t base = (size_t)b * a.bs * width + (size_t)piece * 8;
#pragma unroll 8
            for (int r = 0; r < rows; ++r) {
                Raw8<BF16> x;
                float f[8];
                x.load(a.kc, base + (size_t)r * width);
                x.widen(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    fine &= fabsf(f[e]) <= LARGEST;      // (false for a NaN)
                    lo[e] = fminf(lo[e], f[e]);
                    hi[e] = fmaxf(hi[e], f[e]);
                }
            }
        }
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fmaxf(fabsf(lo[e]), fabsf(hi[e])));
        if (!fine) m = __builtin_inff();
#pragma unroll
        for (int o = 1; o < LPH; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
        if (!on) continue;
        const bool finite = m <= LARGEST;
        const float f = finite && m >= TINY ? 127.f / m : 0.f;
        uint64_t up = 0, down = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int x = finite ? (int)fminf(fmaxf(ceilf(hi[e] * f), -127.f), 127.f) : 0, y = finite ? (int)fminf(fmaxf(floorf(lo[e] * f), -127.f), 127.f) : 0;
            up |= (uint64_t)(uint8_t)x << (8 * e);
            down |= (uint64_t)(uint8_t)y << (8 * e);
        }
        const int head = piece / LPH, d = piece % LPH * 8;
        int8_t *to = a.bounds + ((size_t)b * a.Hkv + head) * 2 * D + d;
        *(uint64_t *)to = up;
        *(uint64_t *)(to + D) = down;
        if (d == 0) a.scales[(size_t)b * a.Hkv + head] = finite ? m / 127.f : __builtin_inff();
    }
}

// ---- selection ------------------------------------------------------------------------------------
struct SelectArgs {
    const void *q;
    const int8_t *bounds;
    const float *scales;
    const int32_t *bt, *seq, *pos;
    int32_t *selected;
    uint32_t *keys;                  // [T][Hkv][max_blocks]
    int T, Hkv, lg_g, n_seqs, max_blocks, bs, n_blocks, budget, n_first, n_recent;
};

// Scores as whole numbers of the same order (a zero has no sign).
constexpr uint32_t KEY_ALWAYS = 0xffffffffu;
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

// Blocks of a row's context, 0 for a row that is out of range.
__device__ __forceinline__ int context_blocks(int seq, int pos, int n_seqs, int max_blocks, int bs)
{
    if (seq < 0 || seq >= n_seqs || pos < 0) return 0;
    return (int)min((long long)pos / bs + 1, (long long)max_blocks);
}

// The 8-bit query of a K/V head, 2 D bytes in LDS: up, then down.  The sums over the heads are made in 64 bits, so that they round the same way in any order.
template <int D, bool BF16>
__device__ __forceinline__ void quantize_query(const SelectArgs &a, int t, int hk, int8_t *to, float *scratch)
{
    const int tid = threadIdx.x, G = 1 << a.lg_g;
    double up = 0., down = 0.;
    if (tid < D) {
        for (int g = 0; g < G; ++g) {
            const size_t at = (((size_t)t * a.Hkv + hk) * G + g) * D + tid;
            const float x = BF16 ? bf16_bits_to_f32(((const bf16_t *)a.q)[at]) : ((const float *)a.q)[at];
            up += x > 0.f ? x : 0.f;
            down += x < 0.f ? x : 0.f;
        }
    }
    const float u = (float)up, v = (float)down;
    float m = fmaxf(u, -v);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    if ((tid & 63) == 0 && tid < D) scratch[tid >> 6] = m;
    __syncthreads();
    m = scratch[0];
    if (D > 64) m = fmaxf(m, scratch[1]);
    const float f = m >= TINY && m <= LARGEST ? 127.f / m : 0.f;
    if (tid < D) {
        const float x = rintf(u * f), y = rintf(v * f);
        to[tid] = (int8_t)(fabsf(x) <= 127.f ? (int)x : 0);      // (a sum that is not finite counts as zero)
        to[D + tid] = (int8_t)(fabsf(y) <= 127.f ? (int)y : 0);
    }
    __syncthreads();
}

// One workgroup per (row, K/V head): scores of all blocks, then the budget-th largest key by its digits of 8 bits from the top, then the list.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void block_select_kernel(SelectArgs a)
{
    __shared__ __attribute__((aligned(16))) int8_t query[2 * D];
    __shared__ float scratch[2];
    __shared__ int histogram[256], wave_sums[4][2], digit, left;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, t = (int)blockIdx.x / a.Hkv, hk = (int)blockIdx.x % a.Hkv;
    const int seq = a.seq[t], pos = a.pos[t], n = context_blocks(seq, pos, a.n_seqs, a.max_blocks, a.bs);
    int32_t *out = a.selected + (size_t)blockIdx.x * a.budget;
    if (n <= a.budget) {
        for (int i = tid; i < a.budget; i += 256) out[i] = i < n ? i : -1;
        return;
    }
    quantize_query<D, BF16>(a, t, hk, query, scratch);
    uint32_t *keys = a.keys + (size_t)blockIdx.x * a.max_blocks;
    const int32_t *bt = a.bt + (size_t)seq * a.max_blocks;
    constexpr int LPB = 2 * D / 16;      // lanes per block, 16 bytes each
    const u32x4 mine = *(const u32x4 *)(query + lane % LPB * 16);
    for (int b0 = w * (64 / LPB); b0 < n; b0 += 256 / LPB) {
        const int b = b0 + lane / LPB, block = b < n ? bt[b] : -1;
        const bool in = (unsigned)block < (unsigned)a.n_blocks;
        int sum = 0;
        float scale = 0.f;
        if (in) {
            const u32x4 x = *(const u32x4 *)(a.bounds + ((size_t)block * a.Hkv + hk) * 2 * D + lane % LPB * 16);
            scale = a.scales[(size_t)block * a.Hkv + hk];
            sum = __builtin_amdgcn_sdot4((int)x.x, (int)mine.x, sum, false);
            sum = __builtin_amdgcn_sdot4((int)x.y, (int)mine.y, sum, false);
            sum = __builtin_amdgcn_sdot4((int)x.z, (int)mine.z, sum, false);
            sum = __builtin_amdgcn_sdot4((int)x.w, (int)mine.w, sum, false);
        }
#pragma unroll
        for (int o = 1; o < LPB; o <<= 1) sum += __shfl_xor(sum, o);
        if (lane % LPB == 0 && b < n) {
            const float score = scale <= LARGEST ? fminf(fmaxf((float)sum * scale, -LARGEST), LARGEST) : LARGEST;
            keys[b] = b < a.n_first || b >= n - a.n_recent ? KEY_ALWAYS : key_of(in ? score : NEG_INF);
        }
    }
    __syncthreads();
    // the budget-th largest key, digit by digit; `left` of those equal to it are taken
    uint32_t prefix = 0;
    int want = a.budget;
    for (int shift = 24; shift >= 0; shift -= 8) {
        histogram[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += 256) {
            const uint32_t k = keys[i];
            if (shift == 24 || k >> (shift + 8) == prefix) atomicAdd(&histogram[k >> shift & 255u], 1);      // (counts: the same in any order)
        }
        __syncthreads();
        const int h = histogram[255 - tid];      // from the largest digit down
        int upto = sum_upto64(h);
        if (lane == 63) wave_sums[w][0] = upto;
        __syncthreads();
        for (int i = 0; i < w; ++i) upto += wave_sums[i][0];
        if (upto >= want && upto - h < want) digit = 255 - tid, left = want - (upto - h);
        __syncthreads();
        prefix = prefix << 8 | (uint32_t)digit;
        want = left;
        __syncthreads();
    }
    // a thread looks through blocks that follow each other, so that ranks are in their order
    const int per = (n + 255) / 256, begin = min(n, tid * per), end = min(n, begin + per);
    int above = 0, equal = 0;
    for (int i = begin; i < end; ++i) above += keys[i] > prefix, equal += keys[i] == prefix;
    int ua = sum_upto64(above), ue = sum_upto64(equal);
    if (lane == 63) wave_sums[w][0] = ua, wave_sums[w][1] = ue;
    __syncthreads();
    for (int i = 0; i < w; ++i) ua += wave_sums[i][0], ue += wave_sums[i][1];
    ua -= above, ue -= equal;
    for (int i = begin; i < end; ++i) {
        const uint32_t k = keys[i];
        if (k > prefix || (k == prefix && ue < want)) out[ua + min(ue, want)] = i;
        ua += k > prefix, ue += k == prefix;
    }
}

// ---- attention over the selected blocks -----------------------------------------------------------
struct SelectedArgs {
    ListArgs list;
    const int32_t *seq, *pos, *selected;
    int budget, parts;
};

// The part of a row's list that workgroup blockIdx.x reads, counted in cache rows: places budget entry x block_size + offset.
struct SelectedItem {
    int t, hk, n, pos, lo, hi;
    const int32_t *bt, *entries;
};
__device__ __forceinline__ SelectedItem selected_item(const SelectedArgs &a, int *scratch)
{
    const ListArgs &g = a.list;
    const int rh = (int)blockIdx.x / a.parts, part = (int)blockIdx.x - rh * a.parts, tid = threadIdx.x;
    SelectedItem it;
    it.t = rh / g.Hkv, it.hk = rh - it.t * g.Hkv;
    const int seq = a.seq[it.t];
    it.pos = a.pos[it.t];
    it.n = context_blocks(seq, it.pos, g.n_seqs, g.max_blocks, g.bs);
    it.bt = g.bt + (size_t)(it.n ? seq : 0) * g.max_blocks;
    it.entries = a.selected + (size_t)rh * a.budget;
    // entries up to the last one in use
    int used = 0;
    if (it.n)
        for (int i = tid; i < a.budget; i += 256)
            if ((unsigned)it.entries[i] < (unsigned)it.n) used = i + 1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) used = max(used, __shfl_xor(used, o));
    if ((tid & 63) == 0) scratch[tid >> 6] = used;
    __syncthreads();
    used = max(max(scratch[0], scratch[1]), max(scratch[2], scratch[3]));
    const long long places = (long long)used * g.bs, per = ((places + a.parts - 1) / a.parts + 31) / 32 * 32;
    it.lo = (int)min(part * per, places);
    it.hi = (int)min(it.lo + per, places);
    return it;
}
__device__ __forceinline__ int selected_slot(const ListArgs &g, const SelectedItem &it, int v)
{
    const int i = v / g.bs, e = it.entries[i], off = v - i * g.bs;
    if ((unsigned)e >= (unsigned)it.n || (i > 0 && e <= it.entries[i - 1]) || (long long)e * g.bs + off > it.pos) return -1;
    return slot_at(g, it.bt, e, off);
}

template <int D, int G, bool BF16>
__global__ __launch_bounds__(256) void selected_vector_kernel(SelectedArgs a)
{
    __shared__ VectorScratch<G, D> scr;
    __shared__ int scratch[4];
    const ListArgs &g = a.list;
    const SelectedItem it = selected_item(a, scratch);
    const auto column_at = [&](int c) { return ((long long)it.t * g.Hq + it.hk * G + c) * D; };
    read_list_vector<D, G, BF16>(
        g, it.hk, scr, it.lo, it.hi, it.hi,
        [&](int v) { return selected_slot(g, it, v); },
        [&](int, int) { return true; },
        column_at,
        [&](int c, int d, float M, float L, float o) {
            if (a.parts > 1) {
                const size_t at = (size_t)blockIdx.x * G + c;
                if (d == 0) *(f32x2 *)(g.ml + 2 * at) = (f32x2){M, L};
                g.o[at * D + d] = o;
                return;
            }
            const float y = L == 0.f ? 0.f : o / L;
            if (BF16) ((bf16_t *)g.out)[column_at(c) + d] = (bf16_t)f32_to_bf16_bits(y);
            else ((float *)g.out)[column_at(c) + d] = y;
        });
}

// The heads of a group are columns of one wavefront; the others of the workgroup copy.
template <int D, bool ONCE>
__global__ __launch_bounds__(256, 2) void selected_matrix_kernel(SelectedArgs a)
{
    __shared__ MatrixTiles<D, 4> lds;
    __shared__ int scratch[4];
    const ListArgs &g = a.list;
    const SelectedItem it = selected_item(a, scratch);
    const int columns = 1 << g.lg_g, col = min((int)threadIdx.x & 31, columns - 1);
    const size_t at = ((size_t)it.t * g.Hq + ((size_t)it.hk << g.lg_g) + col) * D;
    read_list_matrix<D, 4, true, ONCE>(
        g, it.hk, lds, it.lo, it.hi, 0x7fffffff, columns,
        [&](int v) { return selected_slot(g, it, v); },
        [&](int) { return 0xffffffffu; },
        at, at, a.parts > 1 ? (long long)blockIdx.x : -1ll, columns);
}

template <int D, bool BF16>
__global__ __launch_bounds__(256) void selected_merge_kernel(SelectedArgs a)
{
    const ListArgs &g = a.list;
    const int c = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (row, query head)
    if (c >= g.T * g.Hq) return;
    const int G = 1 << g.lg_g;
    combine_parts<D, BF16>(g, (size_t)(c >> g.lg_g) * a.parts, 1, a.parts, G, c & (G - 1), (size_t)c * D);
}

// ---- host -----------------------------------------------------------------------------------------
static int check_select(const alora_attn_dims *d)
{
    const int st = check_attention(d);
    if (st) return st;
    return (long long)d->n_tokens * d->n_q_heads > 0x3fffffffll ? ALORA_ESHAPE : ALORA_OK;
}
static size_t select_bytes(const alora_attn_dims *d) { return (size_t)d->n_tokens * d->n_kv_heads * d->max_blocks * sizeof(uint32_t); }

constexpr int MOST_BUDGET = 1 << 20;

// Parts of every list: workgroups for the whole chip, of at least 256 places.
static int selected_parts(const alora_attn_dims *d, int budget)
{
    const long long lists = (long long)d->n_tokens * d->n_kv_heads, places = (long long)budget * d->block_size;
    if (lists == 0) return 1;
    return (int)std::max(1ll, std::min({(1024 + lists - 1) / lists, (places + 255) / 256, (long long)MAX_PARTS}));
}
static size_t selected_ml_bytes(const alora_attn_dims *d, int parts) { return ((size_t)d->n_tokens * d->n_q_heads * parts * 8 + 255) / 256 * 256; }
static size_t selected_bytes(const alora_attn_dims *d, int parts)
{
    return parts > 1 ? selected_ml_bytes(d, parts) + (size_t)d->n_tokens * d->n_q_heads * parts * d->head_dim * 4 : 0;
}

}  // namespace alora

using namespace alora;

extern "C" {

int alora_block_bounds(const void *k_cache, const int64_t *slot_mapping, int8_t *bounds, float *scales, const alora_bounds_dims *dims, void *hip_stream)
{
    const alora_bounds_dims *d = dims;
    if (!d) return ALORA_EINVAL;
    if (d->dtype != ALORA_F32 && d->dtype != ALORA_BF16) return ALORA_EINVAL;
    if (d->n_rows < 0 || d->n_kv_heads < 1 || d->block_size < 1 || d->n_slots < 0) return ALORA_EINVAL;
    if ((d->head_dim != 64 && d->head_dim != 128) || d->n_slots > 0x7fffffffll || d->n_kv_heads > 1 << 16) return ALORA_ESHAPE;
    if (d->n_rows == 0) return ALORA_OK;
    if (!k_cache || !slot_mapping || !bounds || !scales) return ALORA_EINVAL;
    if (((uintptr_t)k_cache | (uintptr_t)bounds) & 15 || (uintptr_t)slot_mapping & 7 || (uintptr_t)scales & 3) return ALORA_EINVAL;
    BoundsArgs a;
    a.kc = k_cache; a.slot = slot_mapping; a.bounds = bounds; a.scales = scales;
    a.n_rows = d->n_rows; a.Hkv = d->n_kv_heads; a.bs = d->block_size; a.units = (d->n_kv_heads * d->head_dim / 8 + 63) / 64;
    a.n_slots = d->n_slots / d->block_size * d->block_size;
    const auto go = [&](auto kernel, int rows) { launch_kernel(kernel, dim3((unsigned)((d->n_rows + rows - 1) / rows)), dim3(256), 0, (hipStream_t)hip_stream, a); };
    const auto choose = [&](auto head_dim, auto bf16) {
        constexpr int D = decltype(head_dim)::value;
        constexpr bool B = decltype(bf16)::value;
        if (d->n_rows <= 1024) go(block_bounds_kernel<D, B, 2>, 2);
        else go(block_bounds_kernel<D, B, 16>, 16);
    };
    typedef std::integral_constant<int, 128> D128;
    typedef std::integral_constant<int, 64> D64;
    if (d->dtype == ALORA_BF16) d->head_dim == 128 ? choose(D128{}, std::true_type{}) : choose(D64{}, std::true_type{});
    else d->head_dim == 128 ? choose(D128{}, std::false_type{}) : choose(D64{}, std::false_type{});
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

int alora_block_select_workspace_bytes(const alora_attn_dims *dims, size_t *out_bytes)
{
    if (!out_bytes) return ALORA_EINVAL;
    const int st = check_select(dims);
    if (st) return st;
    *out_bytes = select_bytes(dims);
    return ALORA_OK;
}

int alora_block_select(const void *q, const int8_t *bounds, const float *scales, const int32_t *block_tables, const int32_t *token_seq_ids,
                       const int32_t *token_positions, int32_t *selected, int32_t budget, int32_t n_first, int32_t n_recent, const alora_attn_dims *dims,
                       void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int st = check_select(dims);
    if (st) return st;
    if (n_first < 0 || n_recent < 1 || budget > MOST_BUDGET || (long long)n_first + n_recent > budget) return ALORA_EINVAL;
    if (dims->n_tokens == 0) return ALORA_OK;
    const size_t need = select_bytes(dims);
    if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return ALORA_EWORKSPACE;
    if (!q || !bounds || !scales || !block_tables || !token_seq_ids || !token_positions || !selected) return ALORA_EINVAL;
    if (((uintptr_t)q | (uintptr_t)bounds) & 15) return ALORA_EINVAL;
    if (((uintptr_t)scales | (uintptr_t)block_tables | (uintptr_t)token_seq_ids | (uintptr_t)token_positions | (uintptr_t)selected) & 3) return ALORA_EINVAL;
    SelectArgs a;
    a.q = q; a.bounds = bounds; a.scales = scales; a.bt = block_tables; a.seq = token_seq_ids; a.pos = token_positions; a.selected = selected;
    a.keys = (uint32_t *)workspace;
    const ListArgs g = list_args(dims, q, nullptr, nullptr, block_tables, nullptr);
    a.T = g.T; a.Hkv = g.Hkv; a.lg_g = g.lg_g; a.n_seqs = g.n_seqs; a.max_blocks = g.max_blocks; a.bs = g.bs; a.n_blocks = g.n_blocks;
    a.budget = budget; a.n_first = n_first; a.n_recent = n_recent;
    const auto go = [&](auto kernel) { launch_kernel(kernel, dim3((unsigned)a.T * (unsigned)a.Hkv), dim3(256), 0, (hipStream_t)hip_stream, a); };
    const bool bf16 = dims->dtype == ALORA_BF16;
    if (dims->head_dim == 128) bf16 ? go(block_select_kernel<128, true>) : go(block_select_kernel<128, false>);
    else bf16 ? go(block_select_kernel<64, true>) : go(block_select_kernel<64, false>);
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

int alora_selected_attention_workspace_bytes(const alora_attn_dims *dims, int32_t budget, size_t *out_bytes)
{
    if (!out_bytes || budget < 1 || budget > MOST_BUDGET) return ALORA_EINVAL;
    const int st = check_select(dims);
    if (st) return st;
    *out_bytes = selected_bytes(dims, selected_parts(dims, budget));
    return ALORA_OK;
}

int alora_selected_attention(const void *q, const void *k_cache, const void *v_cache, const int32_t *block_tables, const int32_t *token_seq_ids,
                             const int32_t *token_positions, const int32_t *selected, int32_t budget, void *out, const alora_attn_dims *dims,
                             void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int st = check_select(dims);
    if (st) return st;
    if (budget < 1 || budget > MOST_BUDGET) return ALORA_EINVAL;
    if ((long long)budget * dims->block_size > 0x3fffffffll) return ALORA_ESHAPE;
    if (dims->n_tokens == 0) return ALORA_OK;
    const int parts = selected_parts(dims, budget);
    const size_t need = selected_bytes(dims, parts);
    if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return ALORA_EWORKSPACE;
    if (!q || !k_cache || !v_cache || !block_tables || !token_seq_ids || !token_positions || !selected || !out) return ALORA_EINVAL;
    if (((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)out) & 15) return ALORA_EINVAL;
    if (((uintptr_t)block_tables | (uintptr_t)token_seq_ids | (uintptr_t)token_positions | (uintptr_t)selected) & 3) return ALORA_EINVAL;
    SelectedArgs a;
    a.list = list_args(dims, q, k_cache, v_cache, block_tables, out);
    a.seq = token_seq_ids; a.pos = token_positions; a.selected = selected; a.budget = budget; a.parts = parts;
    if (parts > 1) {
        a.list.ml = (float *)workspace;
        a.list.o = (float *)((char *)workspace + selected_ml_bytes(dims, parts));
    }
    const bool bf16 = dims->dtype == ALORA_BF16;
    const dim3 grid((unsigned)dims->n_tokens * (unsigned)dims->n_kv_heads * (unsigned)parts);
    const auto go = [&](auto kernel) { launch_kernel(kernel, grid, dim3(256), 0, (hipStream_t)hip_stream, a); };
    const auto choose = [&](auto head_dim, auto is_bf16) {
        constexpr int D = decltype(head_dim)::value;
        constexpr bool B = decltype(is_bf16)::value;
        if constexpr (B) {
            go(selected_matrix_kernel<D, false>);
        } else switch (a.list.lg_g) {
        case 0: go(selected_vector_kernel<D, 1, B>); break;
        case 1: go(selected_vector_kernel<D, 2, B>); break;
        case 2: go(selected_vector_kernel<D, 4, B>); break;
        default: go(selected_vector_kernel<D, 8, B>); break;
        }
        if (parts > 1)
            launch_kernel(selected_merge_kernel<D, B>, dim3(((unsigned)dims->n_tokens * (unsigned)dims->n_q_heads + 3) / 4), dim3(256), 0, (hipStream_t)hip_stream, a);
    };
    typedef std::integral_constant<int, 128> D128;
    typedef std::integral_constant<int, 64> D64;
    if (bf16) dims->head_dim == 128 ? choose(D128{}, std::true_type{}) : choose(D64{}, std::true_type{});
    else dims->head_dim == 128 ? choose(D128{}, std::false_type{}) : choose(D64{}, std::false_type{});
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

}  // extern "C"
