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
// workgroup looks over ROWS rows of the call for the last ones of their blocks; its wavefronts take those in turn, `units` each.  Bound by the chain of
// slot, rows of the block, store, and by memory where there are many blocks: 256 blocks (5 MB) 5.5 us, 520 (18 MB) 7.2, 4096 blocks of 32 KiB 24, 5.6 TB/s.
template <int D, bool BF16, int ROWS>
__global__ __launch_bounds__(256) void block_bounds_kernel(BoundsArgs a)
{
    constexpr int LPH = D / 8;       // lanes per head
    constexpr int AT_ONCE = 8;       // rows (4, 8, 16: 256 blocks 11.7, 11.6, 11.8 us, 2000 27.2, 25.1, 27.5, 8192 rows of blocks of 64 19.1, 20.0, 22.6)
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
        // (512 rows at a time: behind the last row of a batch padded to a fixed size there is none up to its end)
        int found = -1;
        for (long long j = row0 + 64ll; j < a.n_rows && found < 0; j += 512) {
            int far[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) far[i] = block_of(j + 64 * i + lane < a.n_rows ? a.slot[j + 64 * i + lane] : -1);
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                const unsigned long long any = __builtin_amdgcn_ballot_w64(far[i] >= 0);
                if (any) found = __builtin_amdgcn_readlane(far[i], (int)__builtin_ctzll(any));
            }
        }
        if (!later) next = found;
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
            for (int r = 0; r < rows; r += AT_ONCE) {      // (of fewer rows the last one several times: single loads one after the other would cost more)
                Raw8<BF16> x[AT_ONCE];
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) x[i].load(a.kc, base + (size_t)min(r + i, rows - 1) * width);
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) {
                    float f[8];
                    x[i].widen(f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        fine &= fabsf(f[e]) <= LARGEST;      // (false for a NaN)
                        lo[e] = fminf(lo[e], f[e]);
                        hi[e] = fmaxf(hi[e], f[e]);
                    }
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
    uint32_t *keys;                  // [T][Hkv][key_stride]
    int T, Hkv, lg_g, n_seqs, max_blocks, bs, n_blocks, budget, n_first, n_recent, key_stride;
};

// Scores as whole numbers of the same order (a zero has no sign); 0 is no score's.
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

// The 8-bit query of a K/V head, 2 D bytes in LDS: up, then down.  One wavefront.  The sums over the heads are made in 64 bits, so that they round the
// same way in any order.
template <int D, bool BF16>
__device__ __forceinline__ void quantize_query(const SelectArgs &a, int t, int hk, int8_t *to)
{
    constexpr int E = D / 64;        // components a lane
    const int lane = threadIdx.x & 63, G = 1 << a.lg_g;
    double up[E] = {}, down[E] = {};
    for (int g = 0; g < G; ++g) {
        const size_t at = (((size_t)t * a.Hkv + hk) * G + g) * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = BF16 ? bf16_bits_to_f32(((const bf16_t *)a.q)[at + e]) : ((const float *)a.q)[at + e];
            up[e] += x > 0.f ? x : 0.f;
            down[e] += x < 0.f ? x : 0.f;
        }
    }
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) m = fmaxf(m, fmaxf((float)up[e], -(float)down[e]));
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float f = m >= TINY && m <= LARGEST ? 127.f / m : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float x = rintf((float)up[e] * f), y = rintf((float)down[e] * f);
        to[lane * E + e] = (int8_t)(fabsf(x) <= 127.f ? (int)x : 0);      // (a sum that is not finite counts as zero)
        to[D + lane * E + e] = (int8_t)(fabsf(y) <= 127.f ? (int)y : 0);
    }
}

// N sums over the lanes that share a block's bounds (N lanes of a row), half of them left to a lane after every step: lane i ends with sum i.  The mirrored
// lanes come first, when every lane still has a share of every sum.
template <int CTRL, int BIT, int N>
__device__ __forceinline__ void meet(int (&sum)[16], int lane)
{
    const bool up = lane & BIT;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int keep = up ? sum[i + N] : sum[i], give = up ? sum[i] : sum[i + N];
        sum[i] = keep + __builtin_amdgcn_update_dpp(0, give, CTRL, 0xf, 0xf, true);
    }
}

// The scores of as many blocks as lanes share one, with one head's query: 2 D / 16 lanes hold a block's bounds, 16 bytes each (`mine`: those of the query), lane i of them gets the key of
// block i.  All loads are requested before the first is looked at.  Bound by memory: 223 MB for 200 rows over 94 to 1500 blocks in 51 us, 4.4 TB/s, with the lists (contexts of one
// length, one after the other in the pool, 42: what is ragged starts late, and pieces of 2 KiB lie far apart).  Rows in their order 59; batches of eight blocks, with six workgroups to
// a compute unit instead of five, 2 more; keys and lists in two kernels 5 more.
template <int D, bool ONCE>
__device__ __forceinline__ uint32_t block_keys(const SelectArgs &a, int head, u32x4 mine, const int (&block)[2 * D / 16])
{
    constexpr int LPB = 2 * D / 16;
    const int lane = threadIdx.x & 63, part = lane % LPB;
    u32x4 x[LPB];
#pragma unroll
    for (int i = 0; i < LPB; ++i) {
        x[i] = (u32x4){0u, 0u, 0u, 0u};
        if ((unsigned)block[i] < (unsigned)a.n_blocks) {
            const u32x4 *from = (const u32x4 *)(a.bounds + ((size_t)block[i] * a.Hkv + head) * 2 * D + part * 16);
            x[i] = ONCE ? __builtin_nontemporal_load(from) : *from;
        }
    }
    int b = block[0];
#pragma unroll
    for (int i = 1; i < LPB; ++i) b = part == i ? block[i] : b;
    const bool in = (unsigned)b < (unsigned)a.n_blocks;
    const float scale = in ? a.scales[(size_t)b * a.Hkv + head] : 0.f;
    int sum[16];
#pragma unroll
    for (int i = 0; i < LPB; ++i) {
        sum[i] = __builtin_amdgcn_sdot4((int)x[i].x, (int)mine.x, 0, false);
        sum[i] = __builtin_amdgcn_sdot4((int)x[i].y, (int)mine.y, sum[i], false);
        sum[i] = __builtin_amdgcn_sdot4((int)x[i].z, (int)mine.z, sum[i], false);
        sum[i] = __builtin_amdgcn_sdot4((int)x[i].w, (int)mine.w, sum[i], false);
    }
    if constexpr (LPB == 16) meet<0x140, 8, 8>(sum, lane);      // row_mirror
    meet<0x141, 4, 4>(sum, lane);                               // row_half_mirror
    meet<0x4E, 2, 2>(sum, lane);                                // quad_perm [2,3,0,1]
    meet<0xB1, 1, 1>(sum, lane);                                // quad_perm [1,0,3,2]
    const float score = scale <= LARGEST ? fminf(fmaxf((float)sum[0] * scale, -LARGEST), LARGEST) : LARGEST;
    return key_of(in ? score : NEG_INF);
}

// largest over lanes 0 .. lane
__device__ __forceinline__ uint32_t largest_upto64(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
}

// ---- the list from the keys ----
// n keys, of which the first n_first and the last n_recent blocks' do not count (those are always chosen); n > budget.  The threshold is found by counting: keys
// between the smallest and the largest fall into 2048 bins, the bin it lies in is cut again, until a bin is taken whole or holds one value.
// A thread keeps the keys of PER blocks that follow each other (begin ..), 0 where there is none: ranks are then in the blocks' order.
constexpr int BINS = 2048;
struct __attribute__((aligned(16))) ListScratch {
    int bins[2][BINS], sums[16][2];
    uint32_t ends[16][2], bin, left, inside;
};
template <int NT, int PER>
__device__ __forceinline__ void list_of_keys(const SelectArgs &a, int n, const uint32_t (&key)[PER], int begin, int32_t *out, ListScratch &scr)
{
    constexpr int NW = NT / 64, BPT = BINS / NT;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, c0 = a.n_first, c1 = n - a.n_recent;
    int want = a.budget - a.n_first - a.n_recent;
    uint32_t above = 0xffffffffu, equal = 0;        // chosen: keys above `above`, and `want` of those equal to `equal`
    auto counts = [&](int j) { return begin + j >= c0 && begin + j < c1; };
    if (want > 0) {
        uint32_t low = 0xffffffffu, high = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            low = min(low, counts(j) ? key[j] : 0xffffffffu);
            high = max(high, counts(j) ? key[j] : 0u);
        }
        for (int i = tid; i < BINS; i += NT) scr.bins[0][i] = 0;
        low = ~largest_upto64(~low), high = largest_upto64(high);
        if (lane == 63) scr.ends[w][0] = low, scr.ends[w][1] = high;
        __syncthreads();
        low = 0xffffffffu, high = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) low = min(low, scr.ends[i][0]), high = max(high, scr.ends[i][1]);
        uint32_t span = high - low;                 // keys low .. low + span are looked at
        for (int turn = 0;; turn ^= 1) {
            const int shift = max(0, 32 - (int)__builtin_clz(span | 1u) - 11);
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const uint32_t k = key[j] - low;
                if (counts(j) && k <= span) atomicAdd(&scr.bins[turn][k >> shift], 1);      // (counts: the same in any order)
            }
            for (int i = tid; i < BINS; i += NT) scr.bins[turn ^ 1][i] = 0;
            __syncthreads();
            int mine = 0, h[BPT];
#pragma unroll
            for (int j = 0; j < BPT; ++j) h[j] = scr.bins[turn][BINS - 1 - (tid * BPT + j)], mine += h[j];      // from the largest down
            int upto = sum_upto64(mine);
            if (lane == 63) scr.sums[w][0] = upto;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NW; ++i) upto += i < w ? scr.sums[i][0] : 0;
            int before = upto - mine;
            if (before < want && want <= upto) {
#pragma unroll
                for (int j = 0; j < BPT; ++j) {
                    if (before < want && want <= before + h[j]) scr.bin = (uint32_t)(BINS - 1 - (tid * BPT + j)), scr.left = (uint32_t)(want - before), scr.inside = (uint32_t)h[j];
                    before += h[j];
                }
            }
            __syncthreads();
            want = (int)scr.left;
            low += scr.bin << shift;
            if ((int)scr.inside == want) {          // the whole bin
                above = low - 1, want = 0;          // (keys are above 0)
                break;
            }
            if (shift == 0) {
                above = equal = low;
                break;
            }
            span = (1u << shift) - 1;
        }
    }
    int more = 0, same = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const bool in = begin + j < n, c = counts(j);
        more += in && (!c || key[j] > above);
        same += c && want > 0 && key[j] == equal;
    }
    int um = sum_upto64(more), us = sum_upto64(same);
    if (lane == 63) scr.sums[w][0] = um, scr.sums[w][1] = us;      // (the sums of the bins were read ahead of the last barrier)
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) um += i < w ? scr.sums[i][0] : 0, us += i < w ? scr.sums[i][1] : 0;
    um -= more, us -= same;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const bool in = begin + j < n, c = counts(j), m = in && (!c || key[j] > above), e = c && want > 0 && key[j] == equal;
        if (m || (e && us < want)) out[um + min(us, want)] = begin + j;
        um += m, us += e;
    }
}

// The same for more keys than threads keep: they are read again in every step.
template <int NT>
__device__ __forceinline__ void list_of_many_keys(const SelectArgs &a, int n, const uint32_t *key, int32_t *out, ListScratch &scr)
{
    constexpr int NW = NT / 64, BPT = BINS / NT;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, c0 = a.n_first, c1 = n - a.n_recent;
    int want = a.budget - a.n_first - a.n_recent;
    uint32_t above = 0xffffffffu, equal = 0;
    if (want > 0) {
        uint32_t low = 0, span = 0xffffffffu;
        for (;;) {
            const int shift = max(0, 32 - (int)__builtin_clz(span | 1u) - 11);
            for (int i = tid; i < BINS; i += NT) scr.bins[0][i] = 0;
            __syncthreads();
            for (int i = c0 + tid; i < c1; i += NT) {
                const uint32_t k = key[i] - low;
                if (k <= span) atomicAdd(&scr.bins[0][k >> shift], 1);
            }
            __syncthreads();
            int mine = 0, h[BPT];
#pragma unroll
            for (int j = 0; j < BPT; ++j) h[j] = scr.bins[0][BINS - 1 - (tid * BPT + j)], mine += h[j];
            int upto = sum_upto64(mine);
            if (lane == 63) scr.sums[w][0] = upto;
            __syncthreads();
            for (int i = 0; i < w; ++i) upto += scr.sums[i][0];
            int before = upto - mine;
            if (before < want && want <= upto) {
#pragma unroll
                for (int j = 0; j < BPT; ++j) {
                    if (before < want && want <= before + h[j]) scr.bin = (uint32_t)(BINS - 1 - (tid * BPT + j)), scr.left = (uint32_t)(want - before), scr.inside = (uint32_t)h[j];
                    before += h[j];
                }
            }
            __syncthreads();
            want = (int)scr.left;
            low += scr.bin << shift;
            if ((int)scr.inside == want) {
                above = low - 1, want = 0;
                break;
            }
            if (shift == 0) {
                above = equal = low;
                break;
            }
            span = (1u << shift) - 1;
            __syncthreads();
        }
    }
    int chosen = 0, same_before = 0;                // in the chunks before: a chunk is NT blocks that follow each other
    for (int i0 = 0; i0 < n; i0 += NT) {
        const int i = i0 + tid;
        const bool in = i < n, c = i >= c0 && i < c1;
        const uint32_t k = in ? key[i] : 0u;
        const bool m = in && (!c || k > above), e = in && c && want > 0 && k == equal;
        const unsigned long long bm = __builtin_amdgcn_ballot_w64(m), be = __builtin_amdgcn_ballot_w64(e), under = (1ull << lane) - 1;
        __syncthreads();
        if (lane == 0) scr.sums[w][0] = (int)__builtin_popcountll(bm), scr.sums[w][1] = (int)__builtin_popcountll(be);
        __syncthreads();
        int um = chosen + (int)__builtin_popcountll(bm & under), us = same_before + (int)__builtin_popcountll(be & under);
#pragma unroll
        for (int j = 0; j < NW; ++j) {
            if (j < w) um += scr.sums[j][0], us += scr.sums[j][1];
            chosen += scr.sums[j][0], same_before += scr.sums[j][1];
        }
        if (m || (e && us < want)) out[um + min(us, want)] = i;
    }
}

// All blocks of a context that fits the budget, or of a row that is out of range: true.
template <int NT>
__device__ __forceinline__ bool whole_context(const SelectArgs &a, int n, int32_t *out)
{
    if (n > a.budget) return false;
    for (int i = threadIdx.x; i < a.budget; i += NT) out[i] = i < n ? i : -1;
    return true;
}

// One workgroup per (row, K/V head): block ids to LDS, keys in their place, the list.  7 rows of 157 blocks, fp32, 2 heads: 5.5 us, of which the list is half.
constexpr int MOST_IN_LDS = 17 * 256;
template <int D, bool BF16, bool ONCE>
__global__ __launch_bounds__(256) void block_select_kernel(SelectArgs a, AttnArgs rows, int sorted)
{
    constexpr int LPB = 2 * D / 16, UNITS = 64 / LPB;
    extern __shared__ __attribute__((aligned(16))) int ids[];      // max_blocks, rounded up to LPB
    __shared__ __attribute__((aligned(16))) int8_t query[2 * D];
    __shared__ ListScratch scr;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int t = (int)blockIdx.x / a.Hkv, hk = (int)blockIdx.x % a.Hkv, seq, pos;
    if (sorted) {
        Near near;
        bool together;
        const Turn turn = longest_first<false, false>(rows, sorted, (int)blockIdx.x, scr.bins[0], near, together);
        t = __builtin_amdgcn_readfirstlane(turn.t), hk = turn.hk, seq = __builtin_amdgcn_readfirstlane(turn.seq), pos = __builtin_amdgcn_readfirstlane(turn.pos);
        __syncthreads();
    } else {
        seq = a.seq[t], pos = a.pos[t];
    }
    const int n = context_blocks(seq, pos, a.n_seqs, a.max_blocks, a.bs);
    int32_t *out = a.selected + ((size_t)t * a.Hkv + hk) * a.budget;
    if (whole_context<256>(a, n, out)) return;
    const int32_t *bt = a.bt + (size_t)seq * a.max_blocks;
    const int padded = (n + LPB - 1) / LPB * LPB;
    for (int i = tid; i < padded; i += 256) ids[i] = i < n ? bt[i] : -1;
    if (w == 0) quantize_query<D, BF16>(a, t, hk, query);
    __syncthreads();
    const u32x4 mine = *(const u32x4 *)(query + lane % LPB * 16);
    for (int b0 = (w * UNITS + lane / LPB) * LPB; b0 < padded; b0 += 4 * UNITS * LPB) {      // (whole heads of lanes leave the loop together)
        int block[LPB];
#pragma unroll
        for (int i = 0; i < LPB; ++i) block[i] = ids[b0 + i];
        ids[b0 + lane % LPB] = (int)block_keys<D, ONCE>(a, hk, mine, block);
    }
    __syncthreads();
    const auto list = [&](auto per) {
        constexpr int PER = decltype(per)::value;
        uint32_t key[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = tid * PER + j < n ? (uint32_t)ids[tid * PER + j] : 0u;
        list_of_keys<256, PER>(a, n, key, tid * PER, out, scr);
    };
    if (n <= 3 * 256) list(std::integral_constant<int, 3>{});      // (odd numbers: LDS banks)
    else if (n <= 7 * 256) list(std::integral_constant<int, 7>{});
    else list(std::integral_constant<int, 17>{});
}

// The same in two kernels.  Keys of CHUNK blocks of a row, all heads (whose bounds of a block lie next to each other); then a workgroup per
// (row, head) makes the list.  One row over 8188 blocks, 8 heads (17 MB of bounds): 6.8 us, 2.5 TB/s of which a launch and two dependent loads are most, and 7.1.
constexpr int CHUNK = 64;
template <int D, bool BF16, bool ONCE>
__global__ __launch_bounds__(256) void block_keys_kernel(SelectArgs a)
{
    constexpr int LPB = 2 * D / 16, HEADS = 64 / LPB;
    __shared__ __attribute__((aligned(16))) int8_t query[HEADS][2 * D];
    __shared__ __attribute__((aligned(16))) int ids[CHUNK];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, t = blockIdx.y, h0 = (int)blockIdx.z * HEADS, b0 = (int)blockIdx.x * CHUNK;
    const int seq = a.seq[t], n = context_blocks(seq, a.pos[t], a.n_seqs, a.max_blocks, a.bs);
    if (n <= a.budget || b0 >= n) return;
    if (tid < CHUNK) ids[tid] = b0 + tid < n ? a.bt[(size_t)seq * a.max_blocks + b0 + tid] : -1;
    for (int h = w; h < HEADS; h += 4)
        if (h0 + h < a.Hkv) quantize_query<D, BF16>(a, t, h0 + h, query[h]);
    __syncthreads();
    const int head = lane / LPB;
    const u32x4 mine = *(const u32x4 *)(query[head] + lane % LPB * 16);
    for (int g = w * LPB; g < CHUNK; g += 4 * LPB) {
        int block[LPB];
#pragma unroll
        for (int i = 0; i < LPB; ++i) block[i] = h0 + head < a.Hkv ? ids[g + i] : -1;
        const uint32_t k = block_keys<D, ONCE>(a, h0 + head, mine, block);
        const int b = b0 + g + lane % LPB;
        if (h0 + head < a.Hkv && b < n) a.keys[((size_t)t * a.Hkv + h0 + head) * a.key_stride + b] = k;
    }
}
template <int NT>
__global__ __launch_bounds__(NT) void block_list_kernel(SelectArgs a)
{
    __shared__ ListScratch scr;
    const int tid = threadIdx.x, t = (int)blockIdx.x / a.Hkv, n = context_blocks(a.seq[t], a.pos[t], a.n_seqs, a.max_blocks, a.bs);
    int32_t *out = a.selected + (size_t)blockIdx.x * a.budget;
    if (whole_context<NT>(a, n, out)) return;
    const uint32_t *keys = a.keys + (size_t)blockIdx.x * a.key_stride;
    const auto list = [&](auto per) {
        constexpr int PER = decltype(per)::value;
        uint32_t key[PER];
#pragma unroll
        for (int j = 0; j < PER; j += 4) {      // (four at once: single loads of neighbours that lie in different lanes took 2 of 10 us; the last ones read past n, not past the stride)
            u32x4 x = {0u, 0u, 0u, 0u};
            if (tid * PER + j < n) x = *(const u32x4 *)(keys + tid * PER + j);
#pragma unroll
            for (int i = 0; i < 4; ++i) key[j + i] = tid * PER + j + i < n ? x[i] : 0u;
        }
        list_of_keys<NT, PER>(a, n, key, tid * PER, out, scr);
    };
    if (n <= 4 * NT) list(std::integral_constant<int, 4>{});
    else if (n <= 8 * NT) list(std::integral_constant<int, 8>{});
    else if (n <= 32 * NT) list(std::integral_constant<int, 32>{});
    else list_of_many_keys<NT>(a, n, keys, out, scr);
}

// ---- attention over the selected blocks -----------------------------------------------------------
struct SelectedArgs {
    ListArgs list;
    const int32_t *seq, *pos, *selected;
    int budget, whole, parts;        // the first `whole` lists, of a (row, K/V head) each, are read by one workgroup, the others in parts
};

// The part of a row's list that workgroup blockIdx.x reads, counted in cache rows: places budget entry x block_size + offset.
struct SelectedItem {
    int t, hk, n, pos, lo, hi;
    long long part;      // number of the part whose sums are left, -1: a whole list
    const int32_t *bt, *entries;
};
__device__ __forceinline__ SelectedItem selected_item(const SelectedArgs &a, int *scratch)
{
    const ListArgs &g = a.list;
    const int tid = threadIdx.x, i = (int)blockIdx.x - a.whole, rh = i < 0 ? (int)blockIdx.x : a.whole + i / a.parts, parts = i < 0 ? 1 : a.parts, part = i < 0 ? 0 : i % a.parts;
    SelectedItem it;
    it.part = i < 0 ? -1 : i;
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
#pragma unroll
    for (int i = 0; i < 4; ++i) used = max(used, scratch[i]);
    const long long places = (long long)used * g.bs, per = ((places + parts - 1) / parts + 31) / 32 * 32;
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

template <int D, int G>
__global__ __launch_bounds__(256) void selected_vector_kernel(SelectedArgs a)
{
    __shared__ VectorScratch<G, D> scr;
    __shared__ int scratch[4];
    const ListArgs &g = a.list;
    const SelectedItem it = selected_item(a, scratch);
    const auto column_at = [&](int c) { return ((long long)it.t * g.Hq + it.hk * G + c) * D; };
    read_list_vector<D, G>(
        g, it.hk, scr, it.lo, it.hi, it.hi,
        [&](int v) { return selected_slot(g, it, v); },
        [&](int, int) { return true; },
        column_at,
        [&](int c, int d, float M, float L, float o) {
            if (it.part >= 0) {
                const size_t at = (size_t)it.part * G + c;
                if (d == 0) *(f32x2 *)(g.ml + 2 * at) = (f32x2){M, L};
                g.o[at * D + d] = o;
                return;
            }
            ((float *)g.out)[column_at(c) + d] = L == 0.f ? 0.f : o / L;
        });
}

// The heads of a group are columns of one wavefront; the others of the workgroup copy.  Bound by memory: 200 rows of 1600 places, 1.3 GB of K and V in 222 us, 5.9 TB/s.
// 16 columns to a wavefront (heads of a group are 8 at most) and the weights whole, as two bf16 numbers: the products are no bound here, and the error against 64 bits
// is then that of the result's rounding.
template <int D, bool ONCE>
__global__ __launch_bounds__(256, 2) void selected_matrix_kernel(SelectedArgs a)
{
    __shared__ MatrixTiles<D, 4, 16, 512 / D, 1, 2048> lds;      // 64 KiB of tiles: two workgroups share a CU's LDS
    __shared__ int scratch[4];
    const ListArgs &g = a.list;
    const SelectedItem it = selected_item(a, scratch);
    const int columns = 1 << g.lg_g, col = min((int)threadIdx.x & 15, columns - 1);
    const size_t at = ((size_t)it.t * g.Hq + ((size_t)it.hk << g.lg_g) + col) * D;
    read_list_matrix<ONCE, false>(
        g, it.hk, lds, it.lo, it.hi, 0x7fffffff, columns, false,
        [&](int v) { return selected_slot(g, it, v); },
        [&](int) { return 0xffffffffu; },
        at, at, it.part, columns);
}

template <int D, bool BF16>
__global__ __launch_bounds__(256) void selected_merge_kernel(SelectedArgs a)
{
    const ListArgs &g = a.list;
    const int c = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), list = c >> g.lg_g;      // query head of a list in parts
    if (list >= g.T * g.Hkv - a.whole) return;
    const int G = 1 << g.lg_g;
    combine_parts<D, BF16, 16>(g, (size_t)list * a.parts, 1, a.parts, G, c & (G - 1), (((size_t)a.whole << g.lg_g) + c) * D);
}

// ---- host -----------------------------------------------------------------------------------------
static int check_select(const alora_attn_dims *d)
{
    const int st = check_attention(d);
    if (st) return st;
    // (a grid holds fewer than 2^32 threads in a dimension, and 65535 workgroups in the third)
    return (long long)d->n_tokens * d->n_kv_heads >= 1 << 22 || d->max_blocks > 1 << 28 || d->n_kv_heads > 1 << 16 ? ALORA_ESHAPE : ALORA_OK;
}
// Whether keys and lists are made by kernels of their own.
static bool two_kernels(const alora_attn_dims *d) { return d->max_blocks > MOST_IN_LDS || ((long long)d->n_tokens * d->n_kv_heads < 256 && d->max_blocks > 512); }
static size_t key_stride(const alora_attn_dims *d) { return ((size_t)d->max_blocks + 3) / 4 * 4; }
static size_t select_bytes(const alora_attn_dims *d) { return two_kernels(d) ? (size_t)d->n_tokens * d->n_kv_heads * key_stride(d) * sizeof(uint32_t) : 0; }
// What a call needs is not what one of fewer rows does (those may be the ones that take two kernels, or read lists in parts): the largest need of a call of
// up to so many rows, which is what the sizes' functions give.
static size_t select_bytes_upto(const alora_attn_dims *d)
{
    alora_attn_dims few = *d;
    few.n_tokens = std::min(d->n_tokens, 255 / d->n_kv_heads);      // (the most that take two kernels for their number)
    return std::max(select_bytes(d), select_bytes(&few));
}

constexpr int MOST_BUDGET = 1 << 20;

// Lists are read whole while they fill the chip (512 workgroups: two to a compute unit), the others, behind them, in parts: as many as are done first, by what
// was measured: a turn of workgroups takes 4 us and 0.03 for every place, the second kernel 3, each part 0.1 more.  us, 4, 8, 16, 32 parts of 8 lists of 2048
// places: 18.8, 13.4, 11.5, 11.4.  (Of the fp32 kernel for groups of eight heads the chip holds one to a compute unit.  fp32, 200 rows of 1500 places, heads of 128, us, and K and V at
// 4.9 TB/s: 16/4 heads 226 (250), 32/8 422 (500), 32/4 342 (250), 64/8 614 (500).)
struct ListPlan {
    int whole, parts;      // lists that are read whole; parts of the others
};
static ListPlan plan_lists(const alora_attn_dims *d, int budget)
{
    const int lists = d->n_tokens * d->n_kv_heads, rest = lists % 512;
    const float places = (float)budget * (float)d->block_size;
    int best = 1;
    float least = 4.f + 0.03f * places;
    for (int p = 2; p <= MAX_PARTS; ++p) {
        const float us = (float)((rest * p + 511) / 512) * (4.f + 0.03f * places / (float)p) + 3.f + 0.1f * (float)p;
        if (us < least) least = us, best = p;
    }
    return best > 1 && rest ? ListPlan{lists - rest, best} : ListPlan{lists, 1};
}
static size_t in_parts(const alora_attn_dims *d, const ListPlan &p) { return ((size_t)d->n_tokens * d->n_kv_heads - p.whole) * p.parts * (d->n_q_heads / d->n_kv_heads); }
static size_t selected_ml_bytes(const alora_attn_dims *d, const ListPlan &p) { return (in_parts(d, p) * 8 + 255) / 256 * 256; }
static size_t selected_bytes(const alora_attn_dims *d, const ListPlan &p) { return p.parts > 1 ? selected_ml_bytes(d, p) + in_parts(d, p) * d->head_dim * 4 : 0; }
static size_t selected_bytes_upto(const alora_attn_dims *d, int budget)
{
    alora_attn_dims x = *d;
    size_t most = 0;
    for (; x.n_tokens > 0 && x.n_tokens > d->n_tokens - 512; --x.n_tokens) {      // (the lists left over repeat after 512 rows at most)
        most = std::max(most, selected_bytes(&x, plan_lists(&x, budget)));
        if ((d->n_tokens - x.n_tokens + 1) * (d->n_kv_heads % 512) % 512 == 0) break;
    }
    return most;
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
    if ((d->head_dim != 64 && d->head_dim != 128) || d->n_slots > 0x7fffffffll || d->n_kv_heads > 1 << 16 || d->n_rows > 1 << 27) return ALORA_ESHAPE;
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
        // us, 2, 4, 16 rows of the call to a workgroup, bf16, 8 heads of 128: a row for each of 256 blocks 5.2, 8.1, 26.0, of 1024 7.3, 9.6, 28.5, of 2048 14.5, 14.4,
        // 29.8, of 4096 25.0, 24.0, 31.4; chunks of whole blocks of 1024 rows 6.0, 5.1, 5.1, 2048 6.9, 6.1, 5.1, 8192 20.2, 12.1, 6.1, 65536 115, 62, 25.6 (what
        // starts a workgroup is then most of it).
        if (d->n_rows <= 1024) go(block_bounds_kernel<D, B, 2>, 2);
        else if (d->n_rows <= 4096) go(block_bounds_kernel<D, B, 4>, 4);
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
    *out_bytes = select_bytes_upto(dims);
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
    if (!q || !bounds || !scales || no_table(dims, block_tables) || !token_seq_ids || !token_positions || !selected) return ALORA_EINVAL;
    if (((uintptr_t)q | (uintptr_t)bounds) & 15) return ALORA_EINVAL;
    if (((uintptr_t)scales | (uintptr_t)block_tables | (uintptr_t)token_seq_ids | (uintptr_t)token_positions | (uintptr_t)selected) & 3) return ALORA_EINVAL;
    SelectArgs a;
    a.q = q; a.bounds = bounds; a.scales = scales; a.bt = block_tables; a.seq = token_seq_ids; a.pos = token_positions; a.selected = selected;
    a.keys = (uint32_t *)workspace;
    const ListArgs g = list_args(dims, q, nullptr, nullptr, block_tables, nullptr);
    a.T = g.T; a.Hkv = g.Hkv; a.lg_g = g.lg_g; a.n_seqs = g.n_seqs; a.max_blocks = g.max_blocks; a.bs = g.bs; a.n_blocks = g.n_blocks;
    a.budget = budget; a.n_first = n_first; a.n_recent = n_recent; a.key_stride = (int)key_stride(dims);
    const bool bf16 = dims->dtype == ALORA_BF16;
    const dim3 lists((unsigned)a.T * (unsigned)a.Hkv);
    const bool once = dims->n_tokens <= dims->n_seqs;      // bounds that are read once: non-temporal loads (200 rows over 500 blocks 65.7 | 60.0 us, one over 8188 17.3 | 16.4)
    const auto go = [&](auto head_dim, auto is_bf16) {
        constexpr int D = decltype(head_dim)::value, LPB = D / 8, HEADS = 64 / LPB;
        constexpr bool B = decltype(is_bf16)::value;
        if (!two_kernels(dims)) {
            AttnArgs rows = {};
            rows.bt = a.bt; rows.seq = a.seq; rows.pos = a.pos;
            rows.T = a.T; rows.Hkv = a.Hkv; rows.n_seqs = a.n_seqs; rows.max_blocks = a.max_blocks; rows.bs = a.bs; rows.splits = 1;
            const int runs = (a.T + 255) / 256, sorted = lists.x > 1280 ? (a.T + runs - 1) / runs : 0;
            launch_kernel(once ? block_select_kernel<D, B, true> : block_select_kernel<D, B, false>, lists, dim3(256), (unsigned)((a.max_blocks + LPB - 1) / LPB * LPB) * 4, (hipStream_t)hip_stream, a, rows, sorted);
            return;
        }
        for (int t0 = 0; t0 < dims->n_tokens; t0 += 65535) {      // (a grid's second dimension)
            SelectArgs part = a;
            part.T = std::min(65535, dims->n_tokens - t0);
            part.q = (const char *)a.q + (size_t)t0 * dims->n_q_heads * D * (B ? 2 : 4);
            part.seq = a.seq + t0, part.pos = a.pos + t0, part.keys = a.keys + (size_t)t0 * a.Hkv * a.key_stride;
            launch_kernel(once ? block_keys_kernel<D, B, true> : block_keys_kernel<D, B, false>, dim3((unsigned)(a.max_blocks + CHUNK - 1) / CHUNK, (unsigned)part.T, (unsigned)(a.Hkv + HEADS - 1) / HEADS), dim3(256), 0, (hipStream_t)hip_stream, part);
        }
        launch_kernel(block_list_kernel<1024>, lists, dim3(1024), 0, (hipStream_t)hip_stream, a);
    };
    typedef std::integral_constant<int, 128> D128;
    typedef std::integral_constant<int, 64> D64;
    if (bf16) dims->head_dim == 128 ? go(D128{}, std::true_type{}) : go(D64{}, std::true_type{});
    else dims->head_dim == 128 ? go(D128{}, std::false_type{}) : go(D64{}, std::false_type{});
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

int alora_selected_attention_workspace_bytes(const alora_attn_dims *dims, int32_t budget, size_t *out_bytes)
{
    if (!out_bytes || budget < 1 || budget > MOST_BUDGET) return ALORA_EINVAL;
    const int st = check_select(dims);
    if (st) return st;
    *out_bytes = selected_bytes_upto(dims, budget);
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
    const ListPlan plan = plan_lists(dims, budget);
    const size_t need = selected_bytes(dims, plan);
    if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return ALORA_EWORKSPACE;
    if (!q || !k_cache || !v_cache || no_table(dims, block_tables) || !token_seq_ids || !token_positions || !selected || !out) return ALORA_EINVAL;
    if (((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)out) & 15) return ALORA_EINVAL;
    if (((uintptr_t)block_tables | (uintptr_t)token_seq_ids | (uintptr_t)token_positions | (uintptr_t)selected) & 3) return ALORA_EINVAL;
    SelectedArgs a;
    a.list = list_args(dims, q, k_cache, v_cache, block_tables, out);
    a.seq = token_seq_ids; a.pos = token_positions; a.selected = selected; a.budget = budget; a.whole = plan.whole; a.parts = plan.parts;
    const int lists = dims->n_tokens * dims->n_kv_heads, rest = lists - plan.whole;
    if (rest) {
        a.list.ml = (float *)workspace;
        a.list.o = (float *)((char *)workspace + selected_ml_bytes(dims, plan));
    }
    const bool bf16 = dims->dtype == ALORA_BF16;
    const bool once = dims->n_tokens <= dims->n_seqs;      // contexts that are read once: non-temporal copies (200 rows of 1600 places 242 | 221 us, one row the same)
    const dim3 grid((unsigned)plan.whole + (unsigned)rest * (unsigned)plan.parts);
    const auto go = [&](auto kernel) { launch_kernel(kernel, grid, dim3(256), 0, (hipStream_t)hip_stream, a); };
    const auto choose = [&](auto head_dim, auto is_bf16) {
        constexpr int D = decltype(head_dim)::value;
        constexpr bool B = decltype(is_bf16)::value;
        if constexpr (B) {
            once ? go(selected_matrix_kernel<D, true>) : go(selected_matrix_kernel<D, false>);
        } else switch (a.list.lg_g) {
        case 0: go(selected_vector_kernel<D, 1>); break;
        case 1: go(selected_vector_kernel<D, 2>); break;
        case 2: go(selected_vector_kernel<D, 4>); break;
        default: go(selected_vector_kernel<D, 8>); break;
        }
        if (rest) launch_kernel(selected_merge_kernel<D, B>, dim3((((unsigned)rest << a.list.lg_g) + 3) / 4), dim3(256), 0, (hipStream_t)hip_stream, a);
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
