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

// ---- vector arithmetic, fp32: C columns, positions on the lanes -----------------------------------
// head_dim / 8 lanes share a position, 8 elements each; the groups of lanes of all four wavefronts take positions in turn, each with
// running sums of its own, merged in a fixed order at the end.
//   lo, hi         places of the list this workgroup reads
//   masked_from    places from here on are seen by some columns only: seen(c, place)
//   slot_of(place) place in [lo, hi)
//   q_at(c)        element of q a column begins at, -1: no such column
//   store(c, d, M, L, o) takes column c's maximum, sum of weights and, for element d, unnormalised output
template <int C, int D>
struct VectorScratch {
    static constexpr int WINDOW = 2048;      // places of the list whose slots are in LDS
    int slots[WINDOW];
    float m[4][C], l[4][C], acc[4][C][D];
};

template <int D, int C, class SlotOf, class Seen, class QAt, class Store>
__device__ __forceinline__ void read_list_vector(const ListArgs &a, int hk, VectorScratch<C, D> &scr, int lo, int hi, int masked_from, SlotOf slot_of, Seen seen,
                                                 QAt q_at, Store store)
{
    constexpr int LPP = D / 8, PPW = 64 / LPP, PPI = 4 * PPW, U = 2, BLK = PPI * U, WINDOW = VectorScratch<C, D>::WINDOW;
    static_assert(WINDOW % (2 * BLK) == 0, "whole blocks in a window");
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, grp = lane / LPP, ch = lane % LPP, jl = wave * PPW + grp;
    const size_t width = (size_t)a.Hkv * D, col = (size_t)hk * D + 8 * ch;
    Raw8<false> qr[C];
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
    auto fetch = [&](int j0, Raw8<false> (&kr)[U], Raw8<false> (&vr)[U]) {
        unsigned ok = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * PPI + jl, s = j < hi && j - w0 < WINDOW ? scr.slots[j - w0] : -1;
            kr[u].zero(), vr[u].zero();
            if (s >= 0) {
                ok |= 1u << u;
                kr[u].load(a.kc, (size_t)s * width + col);
                vr[u].load(a.vc, (size_t)s * width + col);
            }
        }
        return ok;
    };
    auto consume = [&](int j0, const Raw8<false> (&kr)[U], const Raw8<false> (&vr)[U], unsigned ok) {
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
                const int j = j0 + u * PPI + jl;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const bool on = (ok >> u & 1u) && (j < masked_from || seen(c, j));      // (worked out again: kept, it costs the other tiles 2 to 3 %)
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[c][e] = on ? fmaf(pw[u][c], vf[e], acc[c][e]) : acc[c][e];
                }
            } else {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[c][e] = fmaf(pw[u][c], vf[e], acc[c][e]);
            }
        }
    };
    for (; w0 < hi; w0 += WINDOW) {
        __syncthreads();
        for (int i = tid; i < WINDOW && w0 + i < hi; i += 256) scr.slots[i] = slot_of(w0 + i);
        __syncthreads();
        const int end = min(hi, w0 + WINDOW);
        Raw8<false> kA[U], vA[U], kB[U], vB[U];
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

// ---- matrix instructions: 32 or 16 columns a wavefront, bf16 ----------------------------------------
// The wavefronts of a workgroup share tiles of 32 places in LDS, which all of them copy and each multiplies with its own columns (32x32x16 or 16x16x32
// products): scores^T = K Q^T leaves a column in two or four lanes, down which the softmax runs, and out^T += V^T P takes the weights from the
// score registers.  Rows of K and V go from global memory straight into LDS, STEP tiles of each per barrier, NB in flight or in use.
// A lane copies 16 bytes of a row; which of the row's 16-byte chunks is turned by the row (XOR), so that neither the reads of K fragments (one
// chunk of 32 or 16 rows) nor the transposing reads of V (chunks of four or eight rows) meet in a bank.
template <int D_, int NW_, int COLS_, int NB_, int STEP_, int WINDOW_>
struct MatrixTiles {
    static constexpr int D = D_, NW = NW_, COLS = COLS_, NB = NB_, STEP = STEP_, WINDOW = WINDOW_;
    static constexpr int PITCH = 2 * D, TILE = 32 * PITCH;      // bytes of a row, of 32
    static constexpr int LPR = D / 8, R = 64 / LPR;             // lanes per row, rows per copy
    static constexpr int GROUPS = 32 / R;                       // copies of a tile
    static constexpr int GPW = GROUPS / NW, IPW = 2 * GPW;      // of which a wavefront makes so many, of K and of V
    static constexpr int SP = PITCH + 16;                       // bytes per column where results are turned around
    static_assert(NB % STEP == 0 && NB > STEP && GPW >= 1 && COLS * SP * NW <= NB * 2 * TILE && WINDOW / 32 % STEP == 0 && NB <= WINDOW / 32, "tiles");
    __attribute__((aligned(1024))) unsigned char tiles[NB * 2 * TILE];
    int slots[WINDOW];
    uint32_t ok[WINDOW / 32], tile_ok[NB];
    __device__ static __forceinline__ uint32_t k_turn(int row) { return D == 128 ? (uint32_t)(row & 15) : (uint32_t)(row >> 1 & 7); }
    __device__ static __forceinline__ uint32_t v_turn(int row) { return (D == 128 ? (uint32_t)(row & 3) << 2 : (uint32_t)(row >> 1 & 1) << 2) ^ (uint32_t)(row >> 2 & 1) << 1; }
};

template <int N> struct FloatsOf;
template <> struct FloatsOf<16> { typedef f32x16 type; };
template <> struct FloatsOf<4> { typedef f32x4 type; };
__device__ __forceinline__ f32x16 multiply(bf16x8 x, bf16x8 y, f32x16 z) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(bf16x8 x, bf16x8 y, f32x4 z) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, z, 0, 0, 0); }

// A weight w in two bf16 numbers: its upper half, and the rest of SPLIT * w, rounded.  Both are above zero wherever w is (the rest is 2^-9 w at least), so that an infinite
// value makes an infinity of either product; rounded to the nearest, or of w itself, the rest would be zero or below it half of the time, and the sum no number.  The factor
// is every weight's and the sum's.  What is lost: half a step (2^-8) of a rest below (2^-7 + 2^-9) w, 1.25 * 2^-15 of w.
constexpr float SPLIT = 1.f + 0x1p-9f;

//   columns        of the workgroup that exist; a wavefront beyond them only copies
//   share          (SHARE, two tiles a step) true, of columns for half of the wavefronts at most: the second half has the first half's, and takes every other tile
//   masked_from    places from here on are seen by some columns only: seen(place) = 32 bits of this lane's column, place a multiple of 32 from lo on
//   q_at, out_at   element of q and out where this lane's column begins (column COLS * wavefront + lane % COLS)
//   part           < 0: rows of out; else number of the part whose sums are left, of room for part_columns columns
// The weights go into the product with V as two bf16 numbers (see SPLIT): their rounding adds nothing to that of the result.  ONCE: rows are not read again
// soon (non-temporal copies).
template <bool ONCE, bool SHARE, class L, class SlotOf, class Seen>
__device__ __forceinline__ void read_list_matrix(const ListArgs &a, int hk, L &lds, int lo, int hi, int masked_from, int columns, bool may_share, SlotOf slot_of,
                                                 Seen seen, size_t q_at, size_t out_at, long long part, int part_columns)
{
    constexpr int D = L::D, NW = L::NW, COLS = L::COLS, NB = L::NB, STEP = L::STEP, TILE = L::TILE, PITCH = L::PITCH, WIN = L::WINDOW / 32;
    constexpr int LG = 64 / COLS;                               // lanes of a column
    constexpr int KD = 8 * LG, KS = D / KD;                     // components a product of scores takes, products
    constexpr int ST = 32 / COLS, NV = 32 / LG;                 // score tiles of 32 places, scores a lane holds: places 4 LG (v / 4) + 4 g + v % 4
    constexpr int PS = 32 / KD;                                 // products per 32 places of V
    constexpr int DT = D / COLS, NA = COLS / LG;                // tiles of the result, components a lane holds of one: COLS t + 4 LG (v / 4) + 4 g + v % 4
    typedef typename FloatsOf<NA>::type Floats;
    typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c16 = lane & 15, li = lane % COLS, g = lane / COLS;
    const bool share = SHARE && may_share;
    const int wc = share && w >= NW / 2 ? w - NW / 2 : w, col = COLS * wc + li;
    const bool col_ok = col < columns, work = COLS * wc < columns;
    const uint32_t tiles_at = (uint32_t)(uintptr_t)(lds_byte *)lds.tiles, row_bytes = (uint32_t)a.Hkv * (uint32_t)PITCH, head = (uint32_t)hk * (uint32_t)PITCH;
    const int c_hi = (hi - lo + 31) >> 5;                       // tiles of this part

    bf16x8 qf[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        u32x4 v = {0u, 0u, 0u, 0u};
        if (col_ok) v = *(const u32x4 *)((const bf16_t *)a.q + q_at + KD * s + 8 * g);
        qf[s] = __builtin_bit_cast(bf16x8, v);
    }
    Floats acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < NA; ++e) acc[t][e] = 0.f;
    float m = M_FLOOR, l = 0.f;
    // over the lanes of a column
    auto column_max = [&](float x) {
        float y, z;
        if (LG == 4) x = fmaxf(x, __shfl_xor(x, 16));
        both_halves(x, y, z);
        return fmaxf(y, z);
    };

    // ---- the window: slots of WIN tiles, and which of their places there are -----------------------
    int win = 0;                                                // first tile of the window
    auto refill = [&](int c) {
        win = c;
        __syncthreads();
        const int end = min(32 * WIN, hi - lo - 32 * c);
        for (int i = tid; i - lane < end; i += 64 * NW) {
            const int s = i < end ? slot_of(lo + 32 * c + i) : -1;
            lds.slots[i] = s;
            const unsigned long long have = __builtin_amdgcn_ballot_w64(s >= 0);
            if ((lane & 31) == 0) lds.ok[i >> 5] = (uint32_t)(lane ? have >> 32 : have);
        }
        __syncthreads();
    };
    // ---- copies -------------------------------------------------------------------------------------
    // (Scalar addresses where a copy's rows lie in one cache block, as block sizes of 4 and more allow, gained nothing: 505 us | 501 where products
    // bound the call, 230 | 243 where memory does.)
    struct Entry {
        int slot[L::GPW];
        uint32_t ok;
    };
    auto lookup = [&](int c) {
        Entry e;
#pragma unroll
        for (int i = 0; i < L::GPW; ++i) e.slot[i] = -1;
        e.ok = 0;
        if (c < c_hi) {
#pragma unroll
            for (int i = 0; i < L::GPW; ++i) e.slot[i] = lds.slots[32 * (c - win) + (w + i * NW) * L::R + lane / L::LPR];
            e.ok = lds.ok[c - win];
        }
        return e;
    };
    const uint32_t chunk = (uint32_t)(lane % L::LPR);
    auto issue = [&](int pair, const Entry &e) {
#pragma unroll
        for (int i = 0; i < L::IPW; ++i) {
            const bool v = i >= L::GPW;                         // K first, then V
            const int group = w + i % L::GPW * NW, row = group * L::R + lane / L::LPR, slot = e.slot[i % L::GPW];
            const uint32_t at = head + ((chunk ^ (v ? L::v_turn(row) : L::k_turn(row))) << 4);
            const void *from = (const char *)(v ? a.vc : a.kc) + (unsigned long long)(uint32_t)slot * row_bytes + at;
            if (slot < 0) from = ab_zero_chunk;
            const uint32_t to = tiles_at + (uint32_t)pair * (2 * TILE) + (v ? TILE : 0) + ((uint32_t)group << 10);
            if constexpr (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" : : "s"(to), "v"(from) : "memory");
            else load_lds16(to, from);
        }
        lds.tile_ok[pair] = e.ok;                               // (the same value from every lane)
    };
    // ---- products -----------------------------------------------------------------------------------
    const uint32_t k_base = (uint32_t)li * PITCH + (((uint32_t)g ^ L::k_turn(li)) << 4);      // row li, chunk LG ks + g (of 16 columns: and row 16 + li)
    const int v_row = 4 * g + (c16 >> 2);
    // 8 bytes of components 4 (c16 % 4) .. of a tile (32 columns: of its half lane / 16 % 2); rows 4 g .. + 3, and 4 LG further on, are the places of a lane's scores
    const uint32_t v_base = (uint32_t)v_row * PITCH + (((uint32_t)((c16 & 3) >> 1) + (LG == 2 ? (uint32_t)(2 * (lane >> 4 & 1)) : 0u)) ^ L::v_turn(v_row)) * 16u + (uint32_t)((c16 & 1) << 3);
    auto consume = [&](int c, int pair) {
        const lds_byte *kb = (const lds_byte *)lds.tiles + pair * (2 * TILE), *vb = kb + TILE;
        Floats st[ST];
#pragma unroll
        for (int t = 0; t < ST; ++t)
#pragma unroll
            for (int e = 0; e < NA; ++e) st[t][e] = 0.f;
        bf16x8 kf[KS][ST];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int t = 0; t < ST; ++t) kf[ks][t] = *(const __attribute__((address_space(3))) bf16x8 *)(kb + (k_base ^ (uint32_t)(ks * LG << 4)) + t * 16 * PITCH);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int t = 0; t < ST; ++t) st[t] = multiply(kf[ks][t], qf[ks], st[t]);
        const uint32_t ok = __builtin_amdgcn_readfirstlane(lds.tile_ok[pair]);
        bf16x8 vf[PS][DT];
#pragma unroll
        for (int s = 0; s < PS; ++s)
#pragma unroll
            for (int t = 0; t < DT; ++t) vf[s][t] = read_tr_frag(vb + (v_base ^ (uint32_t)(t * COLS * 2)) + s * 16 * PITCH, PITCH * LG / 2);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(2);
        float sc[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) sc[v] = st[v / NA][v % NA];
        const int place = lo + 32 * c;
        const bool some = place + 31 >= masked_from;
        uint32_t on = ok;
        if (some || ok != 0xffffffffu) {
            if (some) on &= seen(place);
#pragma unroll
            for (int v = 0; v < NV; ++v) sc[v] = on >> (4 * LG * (v >> 2) + 4 * g + (v & 3)) & 1u ? sc[v] : NEG_INF;
        }
        float mx = fmaxf(sc[0], sc[1]);
#pragma unroll
        for (int v = 2; v < NV; v += 2) mx = fmaxf(fmaxf(mx, sc[v]), sc[v + 1]);
        if (__builtin_amdgcn_ballot_w64(mx * a.scale_log2e > m)) {       // (most tiles of a long list bring no new maximum)
            const float mn = fmaxf(m, column_max(mx) * a.scale_log2e);
            const float corr = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= corr;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int e = 0; e < NA; ++e) acc[t][e] *= corr;
        }
        float ps = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            sc[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[v], a.scale_log2e, -m));
            ps += sc[v];
        }
        l += ps;
        u32x4 pv[PS], pr[PS];
#pragma unroll
        for (int s = 0; s < PS; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = sc[8 * s + 2 * i], y = sc[8 * s + 2 * i + 1];
                const uint32_t ux = __float_as_uint(x), uy = __float_as_uint(y);
                pv[s][i] = __builtin_amdgcn_perm(uy, ux, 0x07060302);
                pr[s][i] = pack_bf16(fmaf(x, SPLIT, -__uint_as_float(ux & 0xffff0000u)), fmaf(y, SPLIT, -__uint_as_float(uy & 0xffff0000u)));
            }
        __builtin_amdgcn_s_setprio(0);
        if (some) {
            // A value that some columns do not see may be anything: what is not finite leaves the product (where it would be multiplied by their zeros)
            // and is added for the columns that do see it.
            bool any = false;
#pragma unroll
            for (int s = 0; s < PS; ++s)
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    const u32x4 x = __builtin_bit_cast(u32x4, vf[s][t]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) any |= (x[i] & 0x7f80u) == 0x7f80u || (x[i] & 0x7f800000u) == 0x7f800000u;
                }
            if (__builtin_amdgcn_ballot_w64(any)) {
#pragma unroll
                for (int s = 0; s < PS; ++s)
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        u32x4 x = __builtin_bit_cast(u32x4, vf[s][t]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if ((x[i] & 0x7f80u) == 0x7f80u) x[i] &= 0xffff0000u;
                            if ((x[i] & 0x7f800000u) == 0x7f800000u) x[i] &= 0xffffu;
                        }
                        vf[s][t] = __builtin_bit_cast(bf16x8, x);
                    }
#pragma unroll 1
                for (int i = 0; i < 32; ++i) {
                    float p = 0.f;              // the column's weight of place i
#pragma unroll
                    for (int v = 0; v < NV; ++v) p = i / (4 * LG) * 4 + (i & 3) == v ? sc[v] : p;
                    p = __shfl(p, li + COLS * (i >> 2 & (LG - 1)));
#pragma unroll
                    for (int t = 0; t < DT; ++t)
#pragma unroll
                        for (int v = 0; v < NA; ++v) {
                            const uint32_t d = (uint32_t)(COLS * t + 4 * LG * (v >> 2) + 4 * g + (v & 3));
                            const float z = bf16_bits_to_f32(*(const __attribute__((address_space(3))) bf16_t *)(vb + i * PITCH + (((d >> 3) ^ L::v_turn(i)) << 4) + (d & 7) * 2));
                            if (!(fabsf(z) <= 3.402823466e38f) && (on >> i & 1u)) acc[t][v] += p * z;      // (seen: however small the weight)
                        }
                }
            }
        }
#pragma unroll
        for (int s = 0; s < PS; ++s)
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                acc[t] = multiply(vf[s][t], __builtin_bit_cast(bf16x8, pv[s]), acc[t]);
                acc[t] = multiply(vf[s][t], __builtin_bit_cast(bf16x8, pr[s]), acc[t]);
            }
    };
    // ---- the list, STEP tiles at a time -------------------------------------------------------------
    // Tile c lives in pair c % NB.  A step waits for its own copies of tiles c .. c + STEP - 1 (those of the NB - 2 STEP behind them stay in flight); the
    // barrier makes that hold for all wavefronts and tells that the step before has been multiplied by everyone: its pairs take the next tiles,
    // whose slots were looked up a step earlier.  Tiles past the list are copied too (zeros), which keeps the count in flight the same.
    if (c_hi > 0) {
        refill(0);
#pragma unroll
        for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[s]));      // (waited for here, not in the loop, where the copies would be waited for too)
#pragma unroll
        for (int k = 0; k < NB - STEP; ++k) issue(k, lookup(k));
        Entry next[STEP];
#pragma unroll
        for (int k = 0; k < STEP; ++k) next[k] = lookup(NB - STEP + k);
        int cur = 0, nxt = NB - STEP;
        const uint32_t mine = !share ? 3u : w < NW / 2 ? 1u : 2u;      // tiles of a step that this wavefront multiplies
        for (int c = 0; c < c_hi; c += STEP) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(L::IPW * (NB - 2 * STEP)) : "memory");
#pragma unroll
            for (int k = 0; k < STEP; ++k) issue(nxt + k, next[k]);
            const int cn = c + NB;
            if (cn == win + WIN && cn < c_hi) refill(cn);
#pragma unroll
            for (int k = 0; k < STEP; ++k) next[k] = lookup(cn + k);
            if (work) {
#pragma unroll
                for (int k = 0; k < STEP; ++k)
                    if ((!SHARE || mine >> k & 1u) && (k == 0 || c + k < c_hi)) consume(c + k, cur + k);
            }
            cur = cur + STEP == NB ? 0 : cur + STEP;
            nxt = nxt + STEP == NB ? 0 : nxt + STEP;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // nothing may be on its way into LDS when the workgroup gives it back
    }
    {
        float x, y;
        if (LG == 4) l += __shfl_xor(l, 16);
        both_halves(l, x, y);
        l = (x + y) * SPLIT;
    }
    if (share) {
        // the second half's sums go to the first half, in a fixed order
        float *const ml = (float *)lds.slots;
        lds_byte *const sums = (lds_byte *)lds.tiles + NB * TILE + wc * (COLS * D * 4);
        static_assert(!SHARE || (STEP == 2 && NW / 2 * COLS * D * 4 <= NB * TILE && NW * COLS * 4 <= (int)sizeof(lds.slots)), "room for the sums, behind that for turning results around");
        __syncthreads();
        if (w >= NW / 2) {
            if (g == 0) ml[2 * col] = m, ml[2 * col + 1] = l;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int v = 0; v < NA; v += 4)
                    *(__attribute__((address_space(3))) f32x4 *)(sums + (((t * NA + v) / 4 * 64 + lane) << 4)) = (f32x4){acc[t][v], acc[t][v + 1], acc[t][v + 2], acc[t][v + 3]};
        }
        __syncthreads();
        if (w >= NW / 2) return;
        const float mo = ml[2 * col], lo2 = ml[2 * col + 1], mn = fmaxf(m, mo), ca = __builtin_amdgcn_exp2f(m - mn), cb = __builtin_amdgcn_exp2f(mo - mn);
        m = mn;
        l = l * ca + lo2 * cb;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < NA; v += 4) {
                const f32x4 x = *(const __attribute__((address_space(3))) f32x4 *)(sums + (((t * NA + v) / 4 * 64 + lane) << 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t][v + e] = acc[t][v + e] * ca + x[e] * cb;
            }
    }
    if (part >= 0) {
        if (col_ok) {
            const size_t at = (size_t)part * part_columns + col;
            if (g == 0) *(f32x2 *)(a.ml + 2 * at) = (f32x2){m, l};
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int v = 0; v < NA; v += 4)
                    *(f32x4 *)(a.o + at * D + COLS * t + LG * v + 4 * g) = (f32x4){acc[t][v], acc[t][v + 1], acc[t][v + 2], acc[t][v + 3]};
        }
        return;
    }
    // columns are rows of the result: a wavefront turns its own around in the tiles, which nobody reads any more
    if (!share) __syncthreads();
    if (!work) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    lds_byte *strip = (lds_byte *)lds.tiles + w * (COLS * L::SP);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int v = 0; v < NA; v += 4)
            *(lds_u32x2 *)(strip + li * L::SP + (COLS * t + LG * v + 4 * g) * 2) =
                (u32x2){pack_bf16(acc[t][v] * inv, acc[t][v + 1] * inv), pack_bf16(acc[t][v + 2] * inv, acc[t][v + 3] * inv)};
#pragma unroll
    for (int i = 0; i < COLS / L::R; ++i) {
        const int c = L::R * i + lane / L::LPR;                 // (a column of this wavefront)
        const u32x4 o = *(const lds_u32x4 *)(strip + c * L::SP + 16 * (lane % L::LPR));
        const size_t at = (size_t)__shfl((unsigned long long)out_at, c);
        if (COLS * w + c < columns) *(u32x4 *)((bf16_t *)a.out + at + 8 * (lane % L::LPR)) = o;
    }
}

// ---- parts of a list, combined --------------------------------------------------------------------
// One wavefront per column: parts first, first + step, ... of `columns` columns each.  head_dim / 4 lanes take a part (four elements each), the others of
// the wavefront the next ones; AHEAD at once.
template <int D, bool BF16, int AHEAD>
__device__ __forceinline__ void combine_parts(const ListArgs &a, size_t first, size_t step, int parts, int columns, int column, size_t out_at)
{
    constexpr int LP = D / 4, NS = 64 / LP;
    const int lane = threadIdx.x & 63, sub = lane / LP, d = lane % LP * 4;
    float M = M_FLOOR, L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = sub; p0 < parts; p0 += NS * AHEAD) {
        f32x2 x[AHEAD];
        f32x4 y[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int p = p0 + NS * i;
            const size_t at = (first + (p < parts ? p : 0) * step) * columns + column;      // (loads without branches)
            x[i] = *(const f32x2 *)(a.ml + 2 * at);
            y[i] = *(const f32x4 *)(a.o + at * D + d);
        }
        float mn = M;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (p0 + NS * i >= parts) x[i] = (f32x2){NEG_INF, 0.f};
            mn = fmaxf(mn, x[i].x);
        }
        const float was = __builtin_amdgcn_exp2f(M - mn);
        M = mn;
        L *= was;
        o *= was;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float f = __builtin_amdgcn_exp2f(x[i].x - mn);
            L += x[i].y * f;
            if (p0 + NS * i < parts) o += y[i] * f;
        }
    }
#pragma unroll
    for (int off = LP; off < 64; off <<= 1) {
        const float mo = __shfl_xor(M, off), lo = __shfl_xor(L, off), mn = fmaxf(M, mo), f = __builtin_amdgcn_exp2f(M - mn), h = __builtin_amdgcn_exp2f(mo - mn);
        M = mn;
        L = L * f + lo * h;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] * f + __shfl_xor(o[e], off) * h;
    }
    if (sub != 0) return;
    const float inv = L == 0.f ? 0.f : 1.f / L;      // (not a number where a weight is none)
    o *= inv;
    if (BF16) *(u32x2 *)((bf16_t *)a.out + out_at + d) = (u32x2){pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    else *(f32x4 *)((float *)a.out + out_at + d) = o;
}

// A table without entries may have no address.
inline bool no_table(const alora_attn_dims *d, const int32_t *block_tables) { return !block_tables && d->n_seqs && d->max_blocks; }

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
