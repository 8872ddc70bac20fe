// Attention of a few columns (query rows x the query heads of one K/V head) over a list of cache positions, which the caller's
// functions spell out: what the readers of drafted trees and of selected blocks have in common.
//
// A list is looked up a window at a time: every thread works out the cache slots of a few places (block table, list of blocks,
// whatever leads there) and leaves them in LDS, -1 where there is nothing to read, so that the loops over the positions know slots
// only.  Parts of a list that several workgroups read leave (maximum, sum of weights, unnormalised output) of every column for
// combine_parts.
#pragma once
#include <type_traits>
#include "alora_attention_core.h"

namespace alora {

constexpr int LIST_WINDOW = 2048;      // places of the list whose slots are in LDS

// What every reader of a list knows.
struct ListArgs {
    const void *q, *kc, *vc;
    void *out;
    const int32_t *bt;
    int T, Hq, Hkv, n_seqs, max_blocks, bs, n_blocks, lg_g;     // n_q_heads / n_kv_heads = 1 << lg_g
    float scale_log2e;                 // scale * log2(e): the softmax runs on powers of two
    float *ml, *o;                     // parts: [part][columns][2], [part][columns][D]
};

// Cache slot of place `at` of block-table row `bt`, -1 where the entry is outside the cache.
__device__ __forceinline__ int slot_at(const ListArgs &a, const int32_t *bt, int block, int offset)
{
    const int b = bt[block];
    return (unsigned)b < (unsigned)a.n_blocks ? b * a.bs + offset : -1;      // (slots are below 2^31)
}

// ---- vector arithmetic: C columns, positions on the lanes -----------------------------------------
// head_dim / 8 lanes share a position, 8 elements each; the groups of lanes of all four wavefronts take positions in turn, each with
// running sums of its own, merged in a fixed order at the end.
//   lo, hi         places of the list this workgroup reads
//   masked_from    places from here on are seen by some columns only: seen(c, place)
//   slot_of(place) place in [lo, hi)
//   q_at(c)        element of q a column begins at, -1: no such column
//   store(c, d, M, L, o) takes column c's maximum, sum of weights and, for element d, unnormalised output
template <int C, int D>
struct VectorScratch {
    int slots[LIST_WINDOW];
    float m[4][C], l[4][C], acc[4][C][D];
};

template <int D, int C, bool BF16, class SlotOf, class Seen, class QAt, class Store>
__device__ __forceinline__ void read_list_vector(const ListArgs &a, int hk, VectorScratch<C, D> &scr, int lo, int hi, int masked_from, SlotOf slot_of, Seen seen,
                                                 QAt q_at, Store store)
{
    constexpr int LPP = D / 8, PPW = 64 / LPP, PPI = 4 * PPW, U = BF16 ? 4 : 2, BLK = PPI * U;
    static_assert(LIST_WINDOW % (2 * BLK) == 0, "whole blocks in a window");
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, grp = lane / LPP, ch = lane % LPP, jl = wave * PPW + grp;
    const size_t width = (size_t)a.Hkv * D, col = (size_t)hk * D + 8 * ch;
    Raw8<BF16> qr[C];
    float m[C], l[C], acc[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const long long at = q_at(c);
        qr[c].zero();
        if (at >= 0) qr[c].load(a.q, (size_t)at + 8 * ch);
        m[c] = M_FLOOR, l[c] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[c][e] = 0.f;
    }
    int w0 = lo;
    auto fetch = [&](int j0, Raw8<BF16> (&kr)[U], Raw8<BF16> (&vr)[U]) {
        unsigned ok = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * PPI + jl, s = j < hi && j - w0 < LIST_WINDOW ? scr.slots[j - w0] : -1;
            kr[u].zero(), vr[u].zero();
            if (s >= 0) {
                ok |= 1u << u;
                kr[u].load(a.kc, (size_t)s * width + col);
                vr[u].load(a.vc, (size_t)s * width + col);
            }
        }
        return ok;
    };
    auto consume = [&](int j0, const Raw8<BF16> (&kr)[U], const Raw8<BF16> (&vr)[U], unsigned ok) {
        float s[U][C];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < C; ++c) s[u][c] = group_sum<LPP>(dot8(qr[c], kr[u]));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * PPI + jl;
#pragma unroll
            for (int c = 0; c < C; ++c) s[u][c] = (ok >> u & 1u) && (j < masked_from || seen(c, j)) ? s[u][c] * a.scale_log2e : NEG_INF;
        }
        float pw[U][C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float mn = m[c];
#pragma unroll
            for (int u = 0; u < U; ++u) mn = fmaxf(mn, s[u][c]);
            const float corr = __builtin_amdgcn_exp2f(m[c] - mn);
            m[c] = mn;
            l[c] *= corr;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                pw[u][c] = __builtin_amdgcn_exp2f(s[u][c] - mn);
                l[c] += pw[u][c];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[c][e] *= corr;
        }
        const bool masked = j0 + BLK > masked_from;     // (a value that a column does not see may be anything)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float vf[8];
            vr[u].widen(vf);
            if (masked) {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[c][e] = pw[u][c] == 0.f ? acc[c][e] : fmaf(pw[u][c], vf[e], acc[c][e]);
            } else {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[c][e] = fmaf(pw[u][c], vf[e], acc[c][e]);
            }
        }
    };
    for (; w0 < hi; w0 += LIST_WINDOW) {
        __syncthreads();
        for (int i = tid; i < LIST_WINDOW && w0 + i < hi; i += 256) scr.slots[i] = slot_of(w0 + i);
        __syncthreads();
        const int end = min(hi, w0 + LIST_WINDOW);
        Raw8<BF16> kA[U], vA[U], kB[U], vB[U];
        unsigned okA = fetch(w0, kA, vA), okB;
        for (int j0 = w0; j0 < end; j0 += 2 * BLK) {
            okB = fetch(j0 + BLK, kB, vB);
            consume(j0, kA, vA, okA);
            okA = fetch(j0 + 2 * BLK, kA, vA);
            consume(j0 + BLK, kB, vB, okB);
        }
    }
#pragma unroll
    for (int off = LPP; off < 64; off <<= 1)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const float mo = __shfl_xor(m[c], off), lo2 = __shfl_xor(l[c], off), mn = fmaxf(m[c], mo);
            const float ca = __builtin_amdgcn_exp2f(m[c] - mn), cb = __builtin_amdgcn_exp2f(mo - mn);
            l[c] = l[c] * ca + lo2 * cb;
            m[c] = mn;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float ao = __shfl_xor(acc[c][e], off);
                acc[c][e] = acc[c][e] * ca + ao * cb;
            }
        }
    if (grp == 0) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (ch == 0) scr.m[wave][c] = m[c], scr.l[wave][c] = l[c];
#pragma unroll
            for (int e = 0; e < 8; ++e) scr.acc[wave][c][8 * ch + e] = acc[c][e];
        }
    }
    __syncthreads();
    for (int i = tid; i < C * D; i += 256) {
        const int c = i / D, d = i % D;
        float M = scr.m[0][c], L = 0.f, o = 0.f;
#pragma unroll
        for (int w = 1; w < 4; ++w) M = fmaxf(M, scr.m[w][c]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(scr.m[w][c] - M);
            L += scr.l[w][c] * f;
            o += scr.acc[w][c][d] * f;
        }
        store(c, d, M, L, o);
    }
}

// ---- parts of a list, combined --------------------------------------------------------------------
// One wavefront per column: parts first, first + step, ... of `columns` columns each.  head_dim / 4 lanes take a part (four elements each), the others of
// the wavefront the next ones.
template <int D, bool BF16>
__device__ __forceinline__ void combine_parts(const ListArgs &a, size_t first, size_t step, int parts, int columns, int column, size_t out_at)
{
    constexpr int LP = D / 4, NS = 64 / LP, AHEAD = 4;
    const int lane = threadIdx.x & 63, sub = lane / LP, d = lane % LP * 4;
    auto ml = [&](int p) { return *(const f32x2 *)(a.ml + 2 * ((first + p * step) * columns + column)); };
    float M = M_FLOOR;
    for (int p = lane; p < parts; p += 64) M = fmaxf(M, ml(p).x);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) M = fmaxf(M, __shfl_xor(M, off));
    float L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = sub; p0 < parts; p0 += NS * AHEAD) {
        f32x2 x[AHEAD];
        f32x4 y[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int p = p0 + NS * i;
            x[i] = (f32x2){M_FLOOR, 0.f};
            y[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
            if (p < parts) {
                x[i] = ml(p);
                y[i] = *(const f32x4 *)(a.o + ((first + p * step) * columns + column) * D + d);
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float f = __builtin_amdgcn_exp2f(x[i].x - M);
            L += x[i].y * f;
            o += y[i] * f;
        }
    }
#pragma unroll
    for (int off = LP; off < 64; off <<= 1) {
        L += __shfl_xor(L, off);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], off);
    }
    if (sub != 0) return;
    const float inv = L == 0.f ? 0.f : 1.f / L;      // (not a number where a weight is none)
    o *= inv;
    if (BF16) *(u32x2 *)((bf16_t *)a.out + out_at + d) = (u32x2){pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    else *(f32x4 *)((float *)a.out + out_at + d) = o;
}

// dims -> what every reader of a list knows (dims checked)
inline ListArgs list_args(const alora_attn_dims *d, const void *q, const void *kc, const void *vc, const int32_t *bt, void *out)
{
    ListArgs a;
    a.q = q; a.kc = kc; a.vc = vc; a.out = out; a.bt = bt;
    a.T = d->n_tokens; a.Hq = d->n_q_heads; a.Hkv = d->n_kv_heads; a.n_seqs = d->n_seqs; a.max_blocks = d->max_blocks; a.bs = d->block_size;
    a.n_blocks = (int)(d->n_slots / d->block_size);
    const int g = d->n_q_heads / d->n_kv_heads;
    a.lg_g = g == 1 ? 0 : g == 2 ? 1 : g == 4 ? 2 : 3;
    a.scale_log2e = (d->scale > 0.f ? d->scale : 1.0f / __builtin_sqrtf((float)d->head_dim)) * 1.4426950408889634f;
    a.ml = a.o = nullptr;
    return a;
}

}  // namespace alora
