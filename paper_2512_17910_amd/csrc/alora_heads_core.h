// What the kernels that turn heads share: how a head lies on lanes, its angles, sums over its lanes (gfx950).
//
// A head's features lie on 2^gshift neighbouring lanes (the first `lanes` of them hold features), each with two chunks of V elements,
// chosen so that no lane needs another's values to turn its own: in halves the chunks at i and i + rot / 2, in neighbours' layout
// two chunks behind each other.  Either way the lane's angles are V consecutive ones of a row of the tables.  The features behind the turned ones
// lie on the lanes behind, two chunks each.  V is 16 bytes of elements where the halves begin at such chunks, else what they allow (a
// chunk that straddles the halves' border would need its partner from two other lanes): 8, 4, 2 for bf16, 4, 2 for fp32.
#pragma once
#include "alora_internal.h"

namespace alora {

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// Workgroups of one dimension of a grid, at most: with 512 threads each they stay below 2^32 threads; further rows go into another dimension.
constexpr int ROWS_AT_ONCE = 1 << 20;

struct HeadShape {
    int d, rot, half;       // features, turned ones, pairs
    int lanes, gshift;      // lanes that hold features; log2 of the lanes of a head
    int interleaved;
};

inline int head_chunk(bool bf16, int rot)   // V
{
    const int half = rot / 2;
    return half % 4 ? 2 : bf16 && half % 8 == 0 ? 8 : 4;
}
// (neighbours' layout needs no border at a chunk: its angles come in fours)
inline int head_chunk(bool bf16, int rot, bool interleaved) { return interleaved && bf16 && rot / 2 % 4 == 0 ? 8 : head_chunk(bf16, rot); }

inline HeadShape head_shape(int d, int rot, bool interleaved, int V)
{
    HeadShape s = {d, rot, rot / 2, 0, 0, interleaved};
    s.lanes = interleaved ? (d + 2 * V - 1) / (2 * V) : s.half / V + (d - rot + 2 * V - 1) / (2 * V);
    while ((1 << s.gshift) < s.lanes) ++s.gshift;
    return s;
}

template <int W>
using Words = uint32_t __attribute__((ext_vector_type(W)));

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
        w = STREAM ? __builtin_nontemporal_load((const Words<W> *)p) : *(const Words<W> *)p;
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void store(char *p) const
    {
        if (STREAM) __builtin_nontemporal_store(w, (Words<W> *)p);
        else *(Words<W> *)p = w;
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
    int a, b, angle;        // elements of the two chunks; first angle
    bool has_a, has_b, turn_a, turn_b;
};
template <int V, bool INTERLEAVED>
__device__ __forceinline__ LanePlace lane_place(const HeadShape &s, int j)
{
    LanePlace p;
    const int pairs = INTERLEAVED ? 0 : s.half / V, rest = j - pairs;
    p.angle = j * V;
    if (INTERLEAVED) {
        p.a = 2 * j * V;
        p.b = p.a + V;
        p.turn_a = p.angle < s.half;
        p.turn_b = p.angle + V / 2 < s.half;    // (angles come in fours, with V = 2 in twos: a chunk is turned whole or not at all)
    } else {
        p.a = rest < 0 ? p.angle : s.rot + 2 * rest * V;
        p.b = rest < 0 ? s.half + p.angle : p.a + V;
        p.turn_a = p.turn_b = rest < 0;
    }
    p.has_a = j < s.lanes && p.a < s.d;
    p.has_b = j < s.lanes && p.b < s.d;
    p.turn_a &= p.has_a;
    p.turn_b &= p.has_b;
    return p;
}

// A lane's V cosines and sines, at row `at` of the tables (element at * half).
template <int V, bool INTERLEAVED>
__device__ __forceinline__ void load_angles(const float *__restrict__ cos, const float *__restrict__ sin, size_t row, const LanePlace &p, float c[V], float s[V])
{
    constexpr int Q = V < 4 ? V : 4;
    typedef float __attribute__((ext_vector_type(Q))) vec;
#pragma unroll
    for (int q = 0; q < V; q += Q) {
        if (INTERLEAVED && q ? p.turn_b : p.turn_a) {
            const vec cv = *(const vec *)(cos + row + p.angle + q), sv = *(const vec *)(sin + row + p.angle + q);
#pragma unroll
            for (int i = 0; i < Q; ++i) { c[q + i] = cv[i]; s[q + i] = sv[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < Q; ++i) { c[q + i] = 1.f; s[q + i] = 0.f; }
        }
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
    ALORA_STEP(5, v[i] + __shfl_xor(v[i], 16))
    ALORA_STEP(6, v[i] + __shfl_xor(v[i], 32))
#undef ALORA_STEP
}

}  // namespace alora
