// A step's rows from lengths on the device (include/alora_steps.h), and what drafted tokens see of their tree (include/alora_tree.h).
#include <algorithm>
#include "alora_steps.h"
#include "alora_tree.h"
#include "alora_attention_internal.h"

namespace alora {

struct StepArgs {
    const int32_t *lengths, *change, *kept, *adapters;
    int32_t *tables, *pool;
    const int32_t *state;
    int32_t *lengths_out, *state_out, *offsets, *seq, *pos, *aid;
    int64_t *slot;
    int n_seqs, max_blocks, bs, row_cap, pool_cap, n_blocks;
};

// Sums over lanes 0 .. lane that stop at LIMIT (operands up to 2^30 + 1 each: no overflow, and min keeps such sums associative).
constexpr unsigned LIMIT = (1u << 30) + 1;
__device__ __forceinline__ unsigned sum_upto64_capped(unsigned x)
{
#define ST_ADD(CTRL, ROWS) x = min(x + (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false), LIMIT)
    ST_ADD(0x111, 0xf);
    ST_ADD(0x112, 0xf);
    ST_ADD(0x114, 0xf);
    ST_ADD(0x118, 0xf);
    ST_ADD(0x142, 0xa);
    ST_ADD(0x143, 0xc);
#undef ST_ADD
    return x;
}

// of the lanes before, from sums over lanes 0 .. lane
__device__ __forceinline__ unsigned sum_before64(unsigned x) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x138, 0xf, 0xf, false); }      // wave_shr:1

constexpr int STEP_SEQS = 256;      // requests looked at together: one a thread

// Largest i with at[i] <= x, of STEP_SEQS ascending entries of which the first is <= x.
__device__ __forceinline__ int find_upto(const unsigned *at, unsigned x)
{
    int i = 0;
#pragma unroll
    for (int step = STEP_SEQS / 2; step; step >>= 1)
        if (at[i + step] <= x) i += step;
    return i;
}

// Three quantities of every request, summed up: blocks it takes, rows it gets, blocks it gives back.  Every workgroup sums them over all requests by
// itself, 256 at a time, and does its share of what they amount to: flat numbers of rows, taken and returned blocks, of which a search in the sums
// tells whose they are.  No workgroup waits for another, and nothing that one reads another writes: new table entries lie behind those read, returned
// blocks go behind the ring entries that are taken.  Bound by the latency of its chain (lengths, two rounds of sums, search, table or ring, store): 64 requests
// of a token 3.9 us, of which a launch is 2.4; 200000 rows (4.2 MB) for 90 requests 6.2; 1.2 million rows 9.4.
__global__ __launch_bounds__(STEP_SEQS) void step_rows_kernel(StepArgs a)
{
    __shared__ unsigned take_at[STEP_SEQS], new_at[STEP_SEQS], back_at[STEP_SEQS], wave_sums[2][4][4];
    __shared__ int len[STEP_SEQS], aid[STEP_SEQS];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const unsigned first_item = blockIdx.x * STEP_SEQS + tid, stride = gridDim.x * STEP_SEQS;
    int first = a.state[0], count = a.state[1];
    if (first < 0 || first >= a.pool_cap || count < 0 || count > a.pool_cap) first = count = 0;
    auto blocks_of = [&](int n) { return (int)(((unsigned)n + (unsigned)a.bs - 1u) / (unsigned)a.bs); };      // (n + block_size - 1 may pass 31 bits)
    auto ring = [&](unsigned i) {       // (first + i with i < pool_cap)
        const unsigned x = (unsigned)first + i;
        return x < (unsigned)a.pool_cap ? x : x - (unsigned)a.pool_cap;
    };
    const long long cap = min((long long)a.max_blocks * a.bs, 0x7fffffffll);
    unsigned asked_blocks = 0, asked_rows = 0, blocks = 0, rows = 0, back = 0, refused = 0;     // of the requests before these
    for (int s0 = 0; s0 < a.n_seqs; s0 += STEP_SEQS) {
        const int s = s0 + tid;
        long long n = 0, c = 0;
        int kept = 0, adapter = -1;
        if (s < a.n_seqs) {
            n = a.lengths[s], c = a.change[s];
            if (a.kept) kept = a.kept[s];
            if (a.adapters) adapter = a.adapters[s];
        }
        const bool valid = n >= 0 && n <= cap && n + c >= 0 && n + c <= cap;
        const int have = valid ? blocks_of((int)n) : 0, want = valid ? (int)((n + c + a.bs - 1) / a.bs) : 0;
        unsigned take = (unsigned)min(max(want - have, 0), (int)LIMIT), fresh = valid ? (unsigned)min(max(c, 0ll), (long long)LIMIT) : 0u;
        // what is asked for decides who is served
        unsigned u = sum_upto64_capped(take), v = sum_upto64_capped(fresh);
        __syncthreads();                 // (the arrays of the requests before are read no more)
        if (lane == 63) wave_sums[0][w][0] = u, wave_sums[0][w][1] = v;
        __syncthreads();
        unsigned bu = asked_blocks, bv = asked_rows;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i == w) u = min(u + bu, LIMIT), v = min(v + bv, LIMIT);
            bu = min(bu + wave_sums[0][i][0], LIMIT), bv = min(bv + wave_sums[0][i][1], LIMIT);
        }
        asked_blocks = bu, asked_rows = bv;
        const bool ok = valid && (c <= 0 || (u <= (unsigned)count && v <= (unsigned)a.row_cap));
        if (!ok) take = fresh = 0;
        const unsigned given = ok ? min((unsigned)max(have - max(want, kept), 0), LIMIT) : 0u;
        // what they get
        const unsigned t1 = sum_upto64_capped(take), f1 = sum_upto64_capped(fresh), g1 = sum_upto64_capped(given);
        const unsigned g0 = sum_before64(g1);      // (a difference would be wrong once the sums stop)
        const unsigned no = (unsigned)__builtin_popcountll(__builtin_amdgcn_ballot_w64(!ok && s < a.n_seqs));
        if (lane == 63) wave_sums[1][w][0] = t1, wave_sums[1][w][1] = f1, wave_sums[1][w][2] = g1, wave_sums[1][w][3] = no;
        __syncthreads();
        unsigned before[4] = {blocks, rows, back, refused}, mine[3] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i == w) mine[0] = before[0] + t1 - take, mine[1] = before[1] + f1 - fresh, mine[2] = min(before[2] + g0, LIMIT);
#pragma unroll
            for (int j = 0; j < 4; ++j) before[j] = min(before[j] + wave_sums[1][i][j], LIMIT);
        }
        take_at[tid] = mine[0], new_at[tid] = mine[1], back_at[tid] = mine[2], len[tid] = (int)n, aid[tid] = adapter;
        if (blockIdx.x == 0 && s < a.n_seqs) {
            a.lengths_out[s] = (int)(ok ? n + c : n);
            a.offsets[s] = (int)mine[1];
        }
        __syncthreads();
        // rows
        for (unsigned r = rows + first_item; r < before[1]; r += stride) {
            const int i = find_upto(new_at, r), p = len[i] + (int)(r - new_at[i]), at = p / a.bs, was = blocks_of(len[i]);
            const int block = at < was ? a.tables[(size_t)(s0 + i) * a.max_blocks + at] : a.pool[ring(take_at[i] + (unsigned)(at - was))];
            a.seq[r] = s0 + i;
            a.pos[r] = p;
            a.aid[r] = aid[i];
            a.slot[r] = block >= 0 && block < a.n_blocks ? (int64_t)block * a.bs + (p - at * a.bs) : -1;
        }
        // blocks taken
        for (unsigned k = blocks + first_item; k < before[0]; k += stride) {
            const int i = find_upto(take_at, k), was = blocks_of(len[i]);
            a.tables[(size_t)(s0 + i) * a.max_blocks + was + (k - take_at[i])] = a.pool[ring(k)];
        }
        // blocks returned, behind those the ring holds, while it has room
        for (unsigned k = back + first_item; k < min(before[2], (unsigned)a.pool_cap - (unsigned)count); k += stride) {
            const int i = find_upto(back_at, k), was = blocks_of(len[i]);
            a.pool[ring((unsigned)count + k)] = a.tables[(size_t)(s0 + i) * a.max_blocks + was - 1 - (int)(k - back_at[i])];
        }
        blocks = before[0], rows = before[1], back = before[2], refused = before[3];
    }
    for (unsigned r = rows + first_item; r < (unsigned)a.row_cap; r += stride) a.seq[r] = a.aid[r] = -1, a.pos[r] = 0, a.slot[r] = -1;
    if (blockIdx.x == 0 && tid == 0) {
        back = min(back, (unsigned)a.pool_cap - (unsigned)count);
        a.offsets[a.n_seqs] = (int)rows;
        a.state_out[0] = a.pool_cap ? (int)ring(blocks == (unsigned)a.pool_cap ? 0u : blocks) : 0;
        a.state_out[1] = count - (int)blocks + (int)back;
        a.state_out[2] = (int)rows;
        a.state_out[3] = (int)blocks;
        a.state_out[4] = (int)back;
        a.state_out[5] = (int)refused;
    }
}

// ---- trees --------------------------------------------------------------------------------------
// One workgroup per sequence, one draft a thread; those behind them clear the rows of no sequence.  Steps to the parent are doubled: after round r a
// draft holds the bits of 2^r ancestors and the place of the next one, so a chain of 255 takes eight rounds, an ordinary tree three.  Bound by latency (two loads, the
// rounds' barriers, a store): 16 trees of up to 25 drafts 3.1 us, 256 of up to 200 4.9; the rows behind all sequences cleared by one workgroup made that 7.1.
template <int WORDS>
__global__ __launch_bounds__(64 * WORDS) void tree_rows_kernel(const int32_t *parents, const int32_t *offsets, const int32_t *context, uint64_t *mask,
                                                               int32_t *pos, int n_tokens, int n_seqs)
{
    constexpr int N = 64 * WORDS;
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= n_seqs) {
        const int begin = n_seqs ? min(max(offsets[0], 0), n_tokens) : 0, end = n_seqs ? min(max(offsets[n_seqs], begin), n_tokens) : 0;
        for (long long t = (long long)((int)blockIdx.x - n_seqs) * N + tid; t < n_tokens; t += (long long)((int)gridDim.x - n_seqs) * N) {
            if (t >= begin && t < end) continue;
            for (int i = 0; i < WORDS; ++i) mask[(size_t)t * WORDS + i] = 0;
            pos[t] = 0;
        }
        return;
    }
    __shared__ uint64_t bits[2][WORDS][N];
    __shared__ int next[2][N];           // the ancestor to go on from, -1: none; -2: an ancestor is not valid
    const int t0 = min(max(offsets[blockIdx.x], 0), n_tokens), rows = min(max(offsets[blockIdx.x + 1], t0), n_tokens) - t0, ctx = context[blockIdx.x];
    uint64_t m[WORDS];
    int to = -1;
    const bool own = tid < rows;
    if (own) {
        to = parents[t0 + tid];
        if (to < -1 || to >= tid) to = -2;
    }
#pragma unroll
    for (int i = 0; i < WORDS; ++i) m[i] = own && tid / 64 == i ? 1ull << (tid & 63) : 0ull;
    for (int round = 0;; round ^= 1) {   // (what a round reads the next but one overwrites: a barrier a round)
#pragma unroll
        for (int i = 0; i < WORDS; ++i) bits[round][i][tid] = m[i];
        next[round][tid] = to;
        if (!__syncthreads_or(to >= 0)) break;
        if (to >= 0) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) m[i] |= bits[round][i][to];
            to = next[round][to];
        }
    }
    if (own) {
        int depth = -1;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if (to == -2) m[i] = 0;
            depth += (int)__builtin_popcountll(m[i]);
            mask[(size_t)(t0 + tid) * WORDS + i] = m[i];
        }
        pos[t0 + tid] = ctx + max(depth, 0);
    }
    for (int t = N + tid; t < rows; t += N) {       // drafts that the masks have no room for
#pragma unroll
        for (int i = 0; i < WORDS; ++i) mask[(size_t)(t0 + t) * WORDS + i] = 0;
        pos[t0 + t] = ctx;
    }
}

static int check_steps(const alora_step_dims *d)
{
    if (!d) return ALORA_EINVAL;
    if (d->n_seqs < 0 || d->max_blocks < 0 || d->block_size < 1 || d->row_cap < 0 || d->pool_cap < 0 || d->n_slots < 0) return ALORA_EINVAL;
    if (d->n_seqs > 1 << 20 || d->row_cap > 1 << 30 || d->pool_cap > 1 << 30 || d->n_slots / d->block_size > 0x7fffffffll) return ALORA_ESHAPE;
    return ALORA_OK;
}

}  // namespace alora

using namespace alora;

extern "C" {

int alora_step_rows(const int32_t *lengths, const int32_t *change, const int32_t *kept_blocks, const int32_t *seq_adapters, int32_t *block_tables,
                    int32_t *pool, const int32_t *state, int32_t *lengths_out, int32_t *state_out, int32_t *row_offsets, int32_t *token_seq_ids,
                    int32_t *token_positions, int32_t *token_adapter_ids, int64_t *slot_mapping, const alora_step_dims *dims, void *hip_stream)
{
    const int st = check_steps(dims);
    if (st) return st;
    if (!state || !state_out || !row_offsets || state_out == state) return ALORA_EINVAL;
    if (dims->n_seqs && (!lengths || !change || !lengths_out || lengths_out == lengths || lengths_out == change)) return ALORA_EINVAL;
    if ((dims->n_seqs && dims->max_blocks && !block_tables) || (dims->pool_cap && !pool)) return ALORA_EINVAL;
    if (dims->row_cap && (!token_seq_ids || !token_positions || !token_adapter_ids || !slot_mapping)) return ALORA_EINVAL;
    if (((uintptr_t)lengths | (uintptr_t)change | (uintptr_t)kept_blocks | (uintptr_t)seq_adapters | (uintptr_t)block_tables | (uintptr_t)pool | (uintptr_t)state |
         (uintptr_t)lengths_out | (uintptr_t)state_out | (uintptr_t)row_offsets | (uintptr_t)token_seq_ids | (uintptr_t)token_positions |
         (uintptr_t)token_adapter_ids) & 3 || (uintptr_t)slot_mapping & 7) return ALORA_EINVAL;
    StepArgs a;
    a.lengths = lengths; a.change = change; a.kept = kept_blocks; a.adapters = seq_adapters;
    a.tables = block_tables; a.pool = pool; a.state = state;
    a.lengths_out = lengths_out; a.state_out = state_out; a.offsets = row_offsets;
    a.seq = token_seq_ids; a.pos = token_positions; a.aid = token_adapter_ids; a.slot = slot_mapping;
    a.n_seqs = dims->n_seqs; a.max_blocks = dims->max_blocks; a.bs = dims->block_size;
    a.row_cap = dims->row_cap; a.pool_cap = dims->pool_cap; a.n_blocks = (int)(dims->n_slots / dims->block_size);
    // Workgroups for half a row or four blocks that may move a thread, at most 1024: each sums all requests by itself, the rest they share.  us, at most 256 | 1024: 64
    // requests that decode 3.9 | 3.9; 40 with 30000 rows each 13.1 | 9.4; 128 of 256 that give back 3750 blocks each 7.4 | 5.5 (by the rows alone, one workgroup, 790).
    const int wgs = std::min(1024, std::max({1, dims->row_cap / 128, dims->pool_cap / 1024}));
    launch_kernel(step_rows_kernel, dim3((unsigned)wgs), dim3(STEP_SEQS), 0, (hipStream_t)hip_stream, a);
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

int alora_tree_rows(const int32_t *tree_parents, const int32_t *row_offsets, const int32_t *context_lens, uint64_t *tree_mask,
                    int32_t *token_positions, int32_t n_tokens, int32_t n_seqs, int32_t mask_words, void *hip_stream)
{
    if (n_tokens < 0 || n_seqs < 0) return ALORA_EINVAL;
    if (mask_words < 1 || mask_words > ALORA_MAX_TREE_WORDS || n_seqs > 1 << 20) return ALORA_ESHAPE;
    if (n_tokens == 0) return ALORA_OK;
    if (!tree_parents || !row_offsets || (n_seqs && !context_lens) || !tree_mask || !token_positions) return ALORA_EINVAL;
    if (((uintptr_t)tree_parents | (uintptr_t)row_offsets | (uintptr_t)context_lens | (uintptr_t)token_positions) & 3 || (uintptr_t)tree_mask & 7) return ALORA_EINVAL;
    const int clearing = (int)std::min(64ll, 1 + n_tokens / (256ll * mask_words));      // workgroups
    const auto go = [&](auto kernel) {
        launch_kernel(kernel, dim3((unsigned)(n_seqs + clearing)), dim3(64 * (unsigned)mask_words), 0, (hipStream_t)hip_stream, tree_parents, row_offsets, context_lens, tree_mask,
                      token_positions, n_tokens, n_seqs);
    };
    mask_words == 1 ? go(tree_rows_kernel<1>) : mask_words == 2 ? go(tree_rows_kernel<2>) : mask_words == 3 ? go(tree_rows_kernel<3>) : go(tree_rows_kernel<4>);
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

}  // extern "C"
