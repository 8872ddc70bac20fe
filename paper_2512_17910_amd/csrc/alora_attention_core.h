// Device functions shared by the readers of the paged cache: pieces of head rows on vector arithmetic, and the copies, fragments and exchanges
// of the kernels on matrix instructions.
#pragma once
#include "alora_attention_internal.h"

namespace alora {

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v)
{
    const int o = __builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true);
    return v + __int_as_float(o);
}

// sum over the LPP lanes that share a position; all of them receive it
template <int LPP>
__device__ __forceinline__ float group_sum(float v)
{
    v = dpp_add<0xB1>(v);    // quad_perm [1,0,3,2]
    v = dpp_add<0x4E>(v);    // quad_perm [2,3,0,1]
    v = dpp_add<0x141>(v);   // row_half_mirror: the other quad of the 8 lanes
    if (LPP == 16) v = dpp_add<0x140>(v);   // row_mirror: the other half of the 16 lanes
    return v;
}

// 8 consecutive elements of a cache or query row, as loaded
template <bool BF16> struct Raw8;
template <> struct Raw8<true> {
    u32x4 v;
    __device__ __forceinline__ void zero() { v = u32x4{0u, 0u, 0u, 0u}; }
    template <bool STREAM = false>
    __device__ __forceinline__ void load(const void *base, size_t elem)
    {
        const u32x4 *p = (const u32x4 *)((const bf16_t *)base + elem);
        v = STREAM ? __builtin_nontemporal_load(p) : *p;
    }
    __device__ __forceinline__ void widen(float f[8]) const
    {
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
        f[4] = __uint_as_float(v.z << 16); f[5] = __uint_as_float(v.z & 0xffff0000u);
        f[6] = __uint_as_float(v.w << 16); f[7] = __uint_as_float(v.w & 0xffff0000u);
    }
};
template <> struct Raw8<false> {
    f32x4 a, b;
    __device__ __forceinline__ void zero() { a = f32x4{0.f, 0.f, 0.f, 0.f}; b = a; }
    template <bool = false>    // (always ordinary loads)
    __device__ __forceinline__ void load(const void *base, size_t elem)
    {
        a = *(const f32x4 *)((const float *)base + elem);
        b = *(const f32x4 *)((const float *)base + elem + 4);
    }
    __device__ __forceinline__ void widen(float f[8]) const
    {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
};

constexpr float NEG_INF = -__builtin_inff();

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

// <q chunk, k chunk> over 8 elements.  bf16: four packed two-element dot products on the stored bits
// (fp32 accumulate); fp32: eight FMAs.  The pairs are taken with shufflevector on the 8-element vector:
// bit casts of the single 32-bit words were compiled into four uses of the first word by this toolchain.
__device__ __forceinline__ float dot8(const Raw8<true> &q, const Raw8<true> &k)
{
    const bf16x8 qv = __builtin_bit_cast(bf16x8, q.v), kv = __builtin_bit_cast(bf16x8, k.v);
    float d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(qv, qv, 0, 1), __builtin_shufflevector(kv, kv, 0, 1), 0.f, false);
    d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(qv, qv, 2, 3), __builtin_shufflevector(kv, kv, 2, 3), d, false);
    d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(qv, qv, 4, 5), __builtin_shufflevector(kv, kv, 4, 5), d, false);
    d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(qv, qv, 6, 7), __builtin_shufflevector(kv, kv, 6, 7), d, false);
    return d;
}
__device__ __forceinline__ float dot8(const Raw8<false> &q, const Raw8<false> &k)
{
    float d = q.a.x * k.a.x;
    d = fmaf(q.a.y, k.a.y, d); d = fmaf(q.a.z, k.a.z, d); d = fmaf(q.a.w, k.a.w, d);
    d = fmaf(q.b.x, k.b.x, d); d = fmaf(q.b.y, k.b.y, d); d = fmaf(q.b.z, k.b.z, d); d = fmaf(q.b.w, k.b.w, d);
    return d;
}

// The running maximum starts at a large negative FINITE number: differences with it stay finite, so the
// softmax needs no "nothing seen yet" cases (a position that is left out scores -inf and weighs
// exp2(-inf) = 0).  Scores below it are treated like -inf.
constexpr float M_FLOOR = -1.0e30f;

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((address_space(3))) unsigned char lds_byte;

constexpr float AB_NEG_INF = -__builtin_inff();
constexpr float AB_M_FLOOR = -1.0e30f;   // finite floor of the running maximum (scores below it weigh nothing)

// four k of this lane's column, then the four that lie eight rows further on
__device__ __forceinline__ bf16x8 read_tr_frag(const lds_byte *p, int pitch)
{
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p + 8 * pitch));
    const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, v);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// 16 bytes straight from global memory into LDS at lds_addr + 16 * lane.  An assembly statement: the
// kernel orders these copies against its LDS reads itself (wait counts and barriers in the main loop).
__device__ __forceinline__ void load_lds16(uint32_t lds_addr, const void *p)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds_addr), "v"(p) : "memory");
}
// the same with a scalar base address and a 32-bit byte offset per lane; ONCE: no other workgroup will read these bytes
template <bool ONCE>
__device__ __forceinline__ void load_lds16(uint32_t lds_addr, const void *base, uint32_t voffset)
{
    if constexpr (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(lds_addr), "v"(voffset), "s"(base) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds_addr), "v"(voffset), "s"(base) : "memory");
}
// Exchange between the two lanes of a column (lanes c, c+32), as an assembly statement (the builtin returned its
// first result twice) with wait states on both sides, which the compiler cannot place for an instruction it does
// not see.  Checked with an in-bounds probe:
//   v_permlane32_swap on two copies of x: lo <- x of the lower 32 lanes, hi <- the upper 32 lanes'
__device__ __forceinline__ void both_halves(float x, float &lo, float &hi)
{
    lo = x, hi = x;
    asm("s_nop 3\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 3" : "+v"(lo), "+v"(hi));
}

// sums of floats, and largest from 0 on, over lanes 0 .. lane
__device__ __forceinline__ float sum_upto64(float x)
{
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x111, 0xf, 0xf, false));
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x112, 0xf, 0xf, false));
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x114, 0xf, 0xf, false));
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x118, 0xf, 0xf, false));
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x142, 0xa, 0xf, false));
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x143, 0xc, 0xf, false));
}
__device__ __forceinline__ int max_upto64(int x)
{
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
    return max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
}

// what a lane loads for a position that is not part of the context (the weighted sum multiplies it by 0)
__device__ const uint32_t ab_zero_chunk[4] = {0u, 0u, 0u, 0u};

// Which row, K/V head and part of the context workgroup b is for when the longest contexts go first; of 256 threads.  Lengths count in
// steps of an eighth (128 of them from 16 positions to a million), rows of one step in batch order: every workgroup finds the same
// order, and each row once.  Where no context is longer than SHORT_CONTEXT, or rows read together (see there), it is the batch's order.  Without parts the order is that
// of every `sorted` rows (at most 256).  In parts there are no more rows than that; those of a.splits parts (see parts_of) come first, where there are
// none the batch's order stays, and the last workgroups find nothing to do (t = -1).  scr: ORDER_SCRATCH ints of LDS.  near: this thread's row.
// GROUPS: look for rows that read together.
struct Turn { int t, seq, pos, hk, part; };
struct Near { int t, seq, n_ctx; };   // a row, its sequence and context (0: none)
constexpr int ORDER_SCRATCH = 128 + 8 + 2;
constexpr int SHORT_CONTEXT = 512;
constexpr int LONG_PART = 512;      // positions per part from which a context is cut into the larger number of parts
__device__ __forceinline__ int parts_of(const AttnArgs &a, int n_ctx) { return n_ctx < a.splits * LONG_PART ? a.short_splits : a.splits; }
template <bool PARTS, bool GROUPS>
__device__ __forceinline__ Turn longest_first(const AttnArgs &a, int sorted, int b, int *scr, Near &near, bool &together)
{
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    unsigned long long *const masks = (unsigned long long *)(scr + 128);
    const int first = PARTS ? 0 : b / a.Hkv / sorted * sorted, rows = min(sorted, a.T - first);
    int key = -1, n_ctx = 0, sq = -1, p = -1;
    bool more = false;
    if (tid < rows) {
        sq = a.seq[first + tid], p = a.pos[first + tid];
        if (sq >= 0 && sq < a.n_seqs && p >= 0) n_ctx = (int)min(p + 1ll, (long long)a.max_blocks * a.bs);
        key = 127 - min(max((int)(__float_as_uint((float)n_ctx) >> 20) - ((127 + 4) << 3), 0), 127);
        more = PARTS && parts_of(a, n_ctx) > a.short_splits;
        if (PARTS) key = (more ? 0 : 64) + (key >> 1);   // (steps of a quarter)
    }
    near = {first + tid, sq, n_ctx};
    if (tid < 128) scr[tid] = 0;
    b -= first * a.Hkv;
    int rank, unit, parts = PARTS ? a.short_splits : 1;
    bool ordered = n_ctx > SHORT_CONTEXT;
    if (PARTS) {
        const int n_more = __syncthreads_count(more), in_more = n_more * a.splits * a.Hkv;
        ordered = n_more > 0;
        if (b < in_more) parts = a.splits;
        else b -= in_more;
        unit = parts * a.Hkv;
        rank = b / unit;
        b -= rank * unit;
        if (parts == a.short_splits) rank += n_more;
        if (rank >= rows) return {-1, -1, -1, 0, 0};
    } else {
        unit = a.Hkv;
        rank = b / unit;
        b -= rank * unit;
    }
    const int hk = b / parts, part = b - hk * parts;
    if (tid == rank) scr[136] = sq, scr[137] = p;
    // Groups of rows that read one context: a row goes with the one before it in the batch if both read the same cache block half way through
    // the shorter of the two.  Where three quarters of the rows are in groups, of eight on average or fewer, the batch's order stays, in which a group
    // reads its context together, with ordinary loads.  us, longest first | batch order: 200 rows that share 1024 of 1075 to 1625 positions in pairs, 8/8
    // heads 184 | 152, 16/8 185 | 155, 32/8 195 | 170 (64/8 265 | 272: not looked for), in fours 8/8 175 | 127, 32/8 186 | 160, in eights 158 | 114 and 171 | 157;
    // half of the rows in pairs 243 | 257 and 260 | 279; a chunk of 144 rows beside 56 others 308 | 333; one prefix for all 196 | 207.
    bool same = false;
    if (GROUPS && tid > 0 && tid < rows) {
        const int sq1 = a.seq[first + tid - 1], half = min(n_ctx, a.pos[first + tid - 1] + 1) >> 1;
        if (half > SHORT_CONTEXT / 2 && sq1 >= 0 && sq1 < a.n_seqs) {
            const int at = a.bs_shift >= 0 ? half >> a.bs_shift : half / a.bs;
            same = a.bt[(size_t)sq * a.max_blocks + at] == a.bt[(size_t)sq1 * a.max_blocks + at];
        }
    }
    const unsigned long long with_last = __builtin_amdgcn_ballot_w64(same);
    const int begin = (int)__builtin_popcountll(with_last & ~(with_last << 1)), in_groups = begin + (int)__builtin_popcountll(with_last);
    if (lane == 0) scr[128 + w] = (__builtin_amdgcn_ballot_w64(ordered) ? 1 << 24 : 0) + (begin << 12) + in_groups;   // (64 and 128 at most)
    __syncthreads();
    const int all = scr[128] + scr[129] + scr[130] + scr[131];
    together = GROUPS && 8 * ((all >> 12) & 0xfff) >= rows && 4 * (all & 0xfff) >= 3 * rows;
    if (all < 1 << 24 || together) return {first + rank, scr[136], scr[137], hk, part};
    if (key >= 0) atomicAdd(&scr[key], 1);   // counts only: their values do not depend on the order
    __syncthreads();
    const int h0 = scr[2 * lane], h1 = scr[2 * lane + 1], upto = sum_upto64(h0 + h1);
    const int at = (int)__builtin_ctzll(__builtin_amdgcn_ballot_w64(rank < upto));   // (rank < rows, the last lane's)
    int n = rank - __builtin_amdgcn_readlane(upto - h0 - h1, at);
    const int even = __builtin_amdgcn_readlane(h0, at), step = 2 * at + (n >= even ? 1 : 0);
    if (n >= even) n -= even;
    const unsigned long long mine = __builtin_amdgcn_ballot_w64(key == step);
    if (lane == 0) masks[w] = mine;
    __syncthreads();
    // the n-th of the step's rows: its thread says which it is
    int before = 0;
    for (int i = 0; i < w; ++i) before += (int)__builtin_popcountll(masks[i]);
    before += __builtin_amdgcn_mbcnt_hi((unsigned)(mine >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mine, 0u));
    if (key == step && before == n) scr[0] = first + tid, scr[136] = sq, scr[137] = p;
    __syncthreads();
    return {scr[0], scr[136], scr[137], hk, part};
}

}  // namespace alora
