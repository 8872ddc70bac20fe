// What the kernels that turn heads share: how a head lies on lanes, its angles, sums over its lanes (gfx950).
//
// A head's features lie on 2^gshift neighbouring lanes (the first `lanes` of them hold features), each with two chunks of V elements,
// chosen so that no lane needs another's values to turn its own, and so that neighbouring lanes' chunks are neighbours in
// memory: a request of the lanes covers whole cache lines.  In halves a lane has the chunks at i and i + rot / 2 and the V angles from i; the
// features behind the turned ones lie on the lanes behind.  In neighbours' layout a pair is inside a chunk: lane j has chunks j and
// j + lanes, and V / 2 angles for each.  V is 16 bytes of elements wherever so much is there.  Where a half, or the features behind, are no
// multiple of V, the last chunk begins earlier and repeats what the one before it has (both lanes compute and store the same values; sums leave
// the repeated elements out): of heads of 80 with 20 turned, 8 lie on a wavefront in bf16 and 4 in fp32, 2 with chunks that divide the half, and
// moves of 9001 bf16 rows of 8 of them over 16 layers take 162 us instead of 334.  Chunks are aligned to 4 bytes, which is all that the loads need.
#pragma once
#include "alora_internal.h"

namespace alora {

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// Workgroups of one dimension of a grid, at most: with 512 threads each they stay below 2^32 threads; further rows go into another dimension.
constexpr int ROWS_AT_ONCE = 1 << 20;

struct HeadShape {
    int d, rot, half;       // features, turned ones, pairs
    int pairs, lanes;       // halves: lanes of turned features; lanes that hold features
    int gshift;             // log2 of the lanes of a head
    int interleaved;
};

inline int head_chunk(bool bf16, int d, int rot, bool interleaved)   // V
{
    if (interleaved) return bf16 && rot % 8 == 0 ? 8 : 4;      // (rot is a multiple of 4)
    int V = bf16 ? 8 : 4;
    while (V > 2 && ((rot && rot / 2 < V) || (rot < d && d - rot < V))) V /= 2;
    return V;
}

inline HeadShape head_shape(int d, int rot, bool interleaved, int V)
{
    HeadShape s = {d, rot, rot / 2, 0, 0, 0, interleaved};
    s.pairs = interleaved ? 0 : (s.half + V - 1) / V;
    s.lanes = interleaved ? (d / V + 1) / 2 : s.pairs + ((d - rot + V - 1) / V + 1) / 2;
    while ((1 << s.gshift) < s.lanes) ++s.gshift;
    return s;
}

template <int W>
using Words = uint32_t __attribute__((ext_vector_type(W)));
template <int W>
using WordsAt4 = uint32_t __attribute__((ext_vector_type(W), aligned(4)));

// V consecutive elements, as they lie in memory
template <bool BF16, int V>
struct Chunk {
    static constexpr int W = BF16 ? V / 2 : V;
    Words<W> w;
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0u;
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void load(const char *p)
    {
        w = STREAM ? __builtin_nontemporal_load((const WordsAt4<W> *)p) : *(const WordsAt4<W> *)p;
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void store(char *p) const
    {
        if (STREAM) __builtin_nontemporal_store(w, (WordsAt4<W> *)p);
        else *(WordsAt4<W> *)p = w;
    }
    __device__ __forceinline__ void widen(float f[V]) const
    {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (BF16) {
                f[2 * i] = __uint_as_float(w[i] << 16);
                f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            } else {
                f[i] = __uint_as_float(w[i]);
            }
        }
    }
    // one rounding, to nearest even
    __device__ __forceinline__ void narrow(const float f[V])
    {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (BF16) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){f[2 * i], f[2 * i + 1]}, bf16x2));
            else w[i] = __float_as_uint(f[i]);
        }
    }
};

// Where a lane's chunks lie in its head, and which of them are turned.
struct LanePlace {
    int a, b;               // elements of the two chunks
    int angle_a, angle_b;   // their first angles (halves: one and the same)
    int again_a, again_b;   // leading elements that another lane's chunk has too
    bool has_a, has_b, turn_a, turn_b;
};
template <int V, bool INTERLEAVED>
__device__ __forceinline__ LanePlace lane_place(const HeadShape &s, int j)
{
    LanePlace p;
    p.has_a = j < s.lanes;
    if (INTERLEAVED) {
        p.a = j * V;
        p.b = (s.lanes + j) * V;
        p.again_a = p.again_b = 0;
        p.has_b = p.has_a && p.b < s.d;
        p.angle_a = p.a / 2;
        p.angle_b = p.b / 2;
        p.turn_a = p.has_a && p.a < s.rot;
        p.turn_b = p.has_b && p.b < s.rot;
    } else if (j < s.pairs) {
        p.a = p.angle_a = p.angle_b = min(j * V, s.half - V);
        p.b = s.half + p.a;
        p.again_a = p.again_b = j * V - p.a;
        p.has_b = p.turn_a = p.turn_b = true;
    } else {
        const int rest = s.d - s.rot, at_a = (j - s.pairs) * V, at_b = at_a + (s.lanes - s.pairs) * V;
        p.a = s.rot + min(at_a, rest - V);
        p.b = s.rot + min(at_b, rest - V);
        p.again_a = s.rot + at_a - p.a;
        p.again_b = s.rot + at_b - p.b;
        p.has_b = p.has_a && at_b < rest;
        p.angle_a = p.angle_b = 0;
        p.turn_a = p.turn_b = false;
    }
    return p;
}

template <int N>
__device__ __forceinline__ void load_floats(const float *p, float *to)
{
    constexpr int Q = N < 4 ? N : 4;
    typedef float __attribute__((ext_vector_type(Q), aligned(4))) vec;
#pragma unroll
    for (int q = 0; q < N; q += Q) {
        const vec v = *(const vec *)(p + q);
#pragma unroll
        for (int i = 0; i < Q; ++i) to[q + i] = v[i];
    }
}

// A lane's V cosines and sines, of the tables' row that begins at element `row`.
template <int V, bool INTERLEAVED>
__device__ __forceinline__ void load_angles(const float *__restrict__ cos, const float *__restrict__ sin, size_t row, const LanePlace &p, float c[V], float s[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) { c[e] = 1.f; s[e] = 0.f; }
    if (INTERLEAVED) {
        if (p.turn_a) {
            load_floats<V / 2>(cos + row + p.angle_a, c);
            load_floats<V / 2>(sin + row + p.angle_a, s);
        }
        if (p.turn_b) {
            load_floats<V / 2>(cos + row + p.angle_b, c + V / 2);
            load_floats<V / 2>(sin + row + p.angle_b, s + V / 2);
        }
    } else if (p.turn_a) {
        load_floats<V>(cos + row + p.angle_a, c);
        load_floats<V>(sin + row + p.angle_a, s);
    }
}

// The lane's features turned by its angles; BACK: by their negatives.  Chunks that are not turned are left alone (a product with a sine of zero
// would carry an infinity over from the other feature).
template <int V, bool INTERLEAVED, bool BACK>
__device__ __forceinline__ void turn(float a[V], float b[V], const float c[V], const float s[V], const LanePlace &p)
{
    if (INTERLEAVED) {
        if (p.turn_a) {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float x = a[2 * i], y = a[2 * i + 1], sn = BACK ? -s[i] : s[i];
                a[2 * i] = x * c[i] - y * sn;
                a[2 * i + 1] = y * c[i] + x * sn;
            }
        }
        if (p.turn_b) {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float x = b[2 * i], y = b[2 * i + 1], cs = c[V / 2 + i], sn = BACK ? -s[V / 2 + i] : s[V / 2 + i];
                b[2 * i] = x * cs - y * sn;
                b[2 * i + 1] = y * cs + x * sn;
            }
        }
    } else if (p.turn_a) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float x = a[i], y = b[i], sn = BACK ? -s[i] : s[i];
            a[i] = x * c[i] - y * sn;
            b[i] = y * c[i] + x * sn;
        }
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp_plus(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// v and the value 16, or 32, lanes away added: the swap exchanges the odd rows of 16 lanes (the upper half) of one copy with the even ones (the lower
// half) of the other, which leaves every lane its own value in one of them and its partner's in the other.
__device__ __forceinline__ float plus_16_away(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float plus_32_away(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// sums over the 2^gshift lanes of a head, N of them side by side; every lane receives them (all 64 lanes take part)
template <int N>
__device__ __forceinline__ void head_sum(float (&v)[N], int gshift)
{
#define ALORA_STEP(bits, value)                    \
    if (gshift >= bits) {                          \
        _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = value; \
    }
    ALORA_STEP(1, dpp_plus<0xB1>(v[i]))    // quad_perm [1,0,3,2]
    ALORA_STEP(2, dpp_plus<0x4E>(v[i]))    // quad_perm [2,3,0,1]
    ALORA_STEP(3, dpp_plus<0x141>(v[i]))   // row_half_mirror: the other quad of the 8 lanes
    ALORA_STEP(4, dpp_plus<0x140>(v[i]))   // row_mirror: the other half of the 16 lanes
    ALORA_STEP(5, plus_16_away(v[i]))
    ALORA_STEP(6, plus_32_away(v[i]))
#undef ALORA_STEP
}

// sums over the lanes that are multiples of 2^gshift apart: of what the heads of a wavefront have in the same place
template <int N>
__device__ __forceinline__ void sum_over_heads(float (&v)[N], int gshift)
{
#define ALORA_STEP(below, value)                    \
    if (gshift < below) {                           \
        _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = value; \
    }
    ALORA_STEP(6, plus_32_away(v[i]))
    ALORA_STEP(5, plus_16_away(v[i]))
    ALORA_STEP(4, dpp_plus<0x128>(v[i]))   // row_ror:8
    ALORA_STEP(3, dpp_plus<0x124>(v[i]))   // row_ror:4, of values that repeat every 8 lanes
    ALORA_STEP(2, dpp_plus<0x122>(v[i]))   // row_ror:2
    ALORA_STEP(1, dpp_plus<0x121>(v[i]))   // row_ror:1
#undef ALORA_STEP
}

}  // namespace alora
