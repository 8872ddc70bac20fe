// Norm of query and key heads with the rotary embedding, in one pass; its backward pass; rotary tables (include/alora_heads.h).
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>
#include "alora_heads.h"
#include "alora_heads_core.h"

namespace alora {

struct HeadsArgs {
    const char *q, *k, *v;
    char *q_out, *kc, *vc;
    const char *wq, *wk;
    const float *cos, *sin;
    const int32_t *pos;
    const int64_t *slot;
    long long q_row, qo_row, k_row, ko_row, v_row, vo_row;   // bytes from row to row
    long long n_slots;
    HeadShape s;
    int T, hq, hkv, n_pos;
    int uq, uk;              // units of 64 >> gshift heads: of queries, of keys
    int items_q, items_k;    // packed rows: wavefronts of queries, of keys
    float eps, inv_d;
};

constexpr int HEADS_WAVES = 8;   // wavefronts of a workgroup, at most

// Pieces of 2 KiB of a row of values: a wavefront's work
__host__ __device__ __forceinline__ int pieces_of(uint32_t bytes) { return (int)(bytes / 2048 + (bytes % 2048 != 0)); }

// U loaded heads of every lane group, normalised, turned and stored where `on`; all 64 lanes take part.
template <bool BF16, int V, bool INTERLEAVED, bool NORM, int U>
__device__ __forceinline__ void norm_turn_store(const HeadsArgs &g, const LanePlace &p, Chunk<BF16, V> (&a)[U], Chunk<BF16, V> (&b)[U],
                                                const Chunk<BF16, V> (&wa)[U], const Chunk<BF16, V> (&wb)[U], const float c[V], const float s[V],
                                                const bool (&on)[U], char *const (&to)[U])
{
    constexpr int E = BF16 ? 2 : 4;
    float r[U];
    if (NORM) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            float x[V], y[V];
            a[i].widen(x);
            b[i].widen(y);
            r[i] = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xe = e < p.again_a ? 0.f : x[e], ye = e < p.again_b ? 0.f : y[e];
                r[i] = fmaf(xe, xe, r[i]);
                r[i] = fmaf(ye, ye, r[i]);
            }
        }
        head_sum<U>(r, g.s.gshift);
#pragma unroll
        for (int i = 0; i < U; ++i) r[i] = rsqrtf(fmaf(r[i], g.inv_d, g.eps));
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        float x[V], y[V];
        a[i].widen(x);
        b[i].widen(y);
        if (NORM) {
            float w[V];
            wa[i].widen(w);
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = x[e] * r[i] * w[e];
            wb[i].widen(w);
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = y[e] * r[i] * w[e];
        }
        turn<V, INTERLEAVED, false>(x, y, c, s, p);
        a[i].narrow(x);
        b[i].narrow(y);
        if (on[i] && p.has_a) a[i].store(to[i] + p.a * E);
        if (on[i] && p.has_b) b[i].store(to[i] + p.b * E);
    }
}

// One workgroup per row: its slot and position are scalars, a lane's angles serve all its heads.  A wavefront takes U units at a time (their
// loads are requested together), the units of queries and keys first, then the row of v in pieces of 2 KiB.  One pass: the mean
// square is a sum over a lane's chunks and over the lanes of the head (DPP), after which the head is still in registers.  Bound by memory: 8192 rows of
// 64 / 8 heads of 128 take 60 us a pass (5.6 TB/s; a large copy reaches 5.2).  Weights loaded behind the sum instead of in front of it, which frees registers: 67.  One row takes 3 us: launch and three dependent loads.
template <bool BF16, int V, bool INTERLEAVED, bool NORM, int U>
__global__ __launch_bounds__(64 * HEADS_WAVES) void heads_kernel(HeadsArgs g)
{
    typedef Chunk<BF16, V> C;
    constexpr int E = BF16 ? 2 : 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    const int gs = g.s.gshift, per = 64 >> gs;
    const LanePlace p = lane_place<V, INTERLEAVED>(g.s, lane & ((1 << gs) - 1));
    const long long row = (long long)blockIdx.y * ROWS_AT_ONCE + blockIdx.x;
    if (row >= g.T) return;
    const long long slot = g.slot[row];
    const bool store = slot >= 0 && slot < g.n_slots;
    const int units = g.uq + g.uk, batches = (units + U - 1) / U;
    const uint32_t v_bytes = g.v ? (uint32_t)g.hkv * g.s.d * E : 0u;      // (rows have at most 2^32 - 16 bytes: a lane's pieces behind them stay below 2^32)
    const int all = batches + pieces_of(v_bytes);

    float c[V], s[V];
    if (g.s.rot && wave < batches) {
        const int at = min(max(g.pos[row], 0), g.n_pos - 1);
        load_angles<V, INTERLEAVED>(g.cos, g.sin, (size_t)at * g.s.half, p, c, s);
    }
    for (int i0 = wave; i0 < all; i0 += waves) {
        if (i0 >= batches) {
            if (!store) break;
            const char *from = g.v + row * g.v_row;
            char *to = g.vc + slot * g.vo_row;
            const uint32_t o = (uint32_t)(i0 - batches) * 2048u + lane * 16;
            u32x4 x, y;
            if (o < v_bytes) x = *(const u32x4 *)(from + o);
            if (o + 1024 < v_bytes) y = *(const u32x4 *)(from + o + 1024);
            if (o < v_bytes) *(u32x4 *)(to + o) = x;
            if (o + 1024 < v_bytes) *(u32x4 *)(to + o + 1024) = y;
            continue;
        }
        C a[U], b[U], wa[U], wb[U];
        char *to[U];
        bool on[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int unit = i0 * U + i;
            const bool is_k = unit >= g.uq;
            const int head = (is_k ? unit - g.uq : unit) * per + (lane >> gs);
            const long long offset = (long long)head * (g.s.d * E);
            on[i] = is_k ? store && head < g.hkv : head < g.hq;    // (units behind the last have no such head)
            const char *from = is_k ? (g.k ? g.k + row * g.k_row : g.kc + slot * g.ko_row) : g.q + row * g.q_row;
            to[i] = (is_k ? g.kc + slot * g.ko_row : g.q_out + row * g.qo_row) + offset;
            a[i].zero();
            b[i].zero();
            if (on[i] && p.has_a) a[i].load(from + offset + p.a * E);
            if (on[i] && p.has_b) b[i].load(from + offset + p.b * E);
            if (NORM) {
                const char *w = is_k ? g.wk : g.wq;
                wa[i].zero();
                wb[i].zero();
                if (p.has_a) wa[i].load(w + p.a * E);
                if (p.has_b) wb[i].load(w + p.b * E);
            }
        }
        norm_turn_store<BF16, V, INTERLEAVED, NORM, U>(g, p, a, b, wa, wb, c, s, on, to);
    }
}

// The same for rows of few heads (at most half a unit): a wavefront takes several rows' queries, keys or values, since what such calls cost is the number of
// wavefronts.  8192 rows of 4 / 1 heads of 64 take 4.9 us, a workgroup for each row 14.0.
template <bool BF16, int V, bool INTERLEAVED, bool NORM>
__global__ __launch_bounds__(256) void heads_packed_kernel(HeadsArgs g)
{
    typedef Chunk<BF16, V> C;
    constexpr int E = BF16 ? 2 : 4;
    const int lane = threadIdx.x & 63;
    int item = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= g.items_q + g.items_k) {      // values: 2 KiB
        item -= g.items_q + g.items_k;
        const int pieces = g.hkv * g.s.d * E / 16, rows = 128 / pieces;
        u32x4 x[2];
        char *to[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = 64 * i + lane, sub = at / pieces, piece = at - sub * pieces;
            const long long row = (long long)item * rows + sub;
            to[i] = nullptr;
            if (g.v && sub < rows && row < g.T) {
                const long long slot = g.slot[row];
                if (slot >= 0 && slot < g.n_slots) {
                    x[i] = *(const u32x4 *)(g.v + row * g.v_row + piece * 16);
                    to[i] = g.vc + slot * g.vo_row + piece * 16;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (to[i]) *(u32x4 *)to[i] = x[i];
        return;
    }
    const bool is_k = item >= g.items_q;
    if (is_k) item -= g.items_q;
    const int gs = g.s.gshift, heads = is_k ? g.hkv : g.hq, rows = (64 >> gs) / heads;
    const LanePlace p = lane_place<V, INTERLEAVED>(g.s, lane & ((1 << gs) - 1));
    const int sub = (lane >> gs) / heads, head = (lane >> gs) - sub * heads;
    const long long row = (long long)item * rows + sub;
    bool on[1] = {sub < rows && row < g.T};
    long long slot = 0;
    if (is_k && on[0]) {
        slot = g.slot[row];
        on[0] = slot >= 0 && slot < g.n_slots;
    }
    C a[1], b[1], wa[1], wb[1];
    a[0].zero(); b[0].zero(); wa[0].zero(); wb[0].zero();
    char *to[1] = {nullptr};
    float c[V], s[V];
    const char *w = is_k ? g.wk : g.wq;
    if (on[0]) {
        const long long offset = (long long)head * (g.s.d * E);
        const char *from = (is_k ? (g.k ? g.k + row * g.k_row : g.kc + slot * g.ko_row) : g.q + row * g.q_row) + offset;
        to[0] = (is_k ? g.kc + slot * g.ko_row : g.q_out + row * g.qo_row) + offset;
        if (p.has_a) a[0].load(from + p.a * E);
        if (p.has_b) b[0].load(from + p.b * E);
        if (g.s.rot) load_angles<V, INTERLEAVED>(g.cos, g.sin, (size_t)min(max(g.pos[row], 0), g.n_pos - 1) * g.s.half, p, c, s);
    }
    if (NORM) {
        if (p.has_a) wa[0].load(w + p.a * E);
        if (p.has_b) wb[0].load(w + p.b * E);
    }
    norm_turn_store<BF16, V, INTERLEAVED, NORM, 1>(g, p, a, b, wa, wb, c, s, on, to);
}

struct HeadsBackArgs {
    const char *q, *k, *gq, *gk;
    char *dq, *dk;
    const char *wq, *wk;
    const float *cos, *sin;
    const int32_t *pos;
    long long q_row, k_row, gq_row, gk_row, dq_row, dk_row;
    float *partial;          // [workgroups][2][d]
    float *dwq, *dwk;        // where one workgroup does it all, it writes these
    HeadShape s;
    int T, hq, hkv, n_pos;
    int rows_q, rows_k;      // rows of a unit: several where their heads are at most half of it
    int uq, uk, wq_waves;    // the first wq_waves wavefronts of a workgroup take the queries
    float eps, inv_d;
};

constexpr int BACK_WAVES = 16;   // wavefronts of a workgroup, at most

// With g = the outputs' gradient turned back, u = g w, r = 1 / sqrt(mean x^2 + eps): both means (of x x and x u) come out of one pass over x and g, then
// dx = r (u - x r (r mean(x u))) from registers (r^3 would leave fp32's range for heads of 1e-13), and each lane adds g x r to sums for the weights of its features.
// The units of heads of all rows, those of queries dealt to the wavefronts of all workgroups that take queries, those of keys to
// the others, so that a lane's sums for the weights are of one of the two.  Bound by memory: 4096 rows of 32 / 8 heads of 128 take 24.5 us (5.2 TB/s),
// the second kernel 4.5, both under the profiler, and the pass of both 28.3.  What was compared when this was chosen, passes of that time: 256 workgroups
// of up to 16 wavefronts (fewer partial sums to add) 27.6, with 512 29.9, 1024 of five wavefronts that kept to rows 42; ordinary stores in place of dx
// past the caches 29.2.  Rows of few heads share a wavefront: 2869 rows of 8 / 1
// heads of 32 take 6.5 us, with a row for each 9.3 (11.0 with the sums over the heads through LDS).
template <bool BF16, int V, bool INTERLEAVED, bool NORM>
__global__ __launch_bounds__(64 * BACK_WAVES) void heads_back_kernel(HeadsBackArgs g)
{
    typedef Chunk<BF16, V> C;
    constexpr int E = BF16 ? 2 : 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    const int gs = g.s.gshift, per = 64 >> gs;
    const LanePlace p = lane_place<V, INTERLEAVED>(g.s, lane & ((1 << gs) - 1));
    const bool is_k = wave >= g.wq_waves;
    const int heads = is_k ? g.hkv : g.hq, units = is_k ? g.uk : g.uq, rows = is_k ? g.rows_k : g.rows_q, T = (g.T + rows - 1) / rows;
    const int mine = is_k ? waves - g.wq_waves : g.wq_waves, step = gridDim.x * mine;
    const int first = blockIdx.x * mine + (is_k ? wave - g.wq_waves : wave);
    const int row_step = step / units, unit_step = step % units;
    const char *xs = is_k ? g.k : g.q, *gs_in = is_k ? g.gk : g.gq;
    char *outs = is_k ? g.dk : g.dq;
    const long long x_row = is_k ? g.k_row : g.q_row, g_row = is_k ? g.gk_row : g.gq_row, d_row = is_k ? g.dk_row : g.dq_row;

    // (several rows of few heads on a wavefront: the lane's row among them, and what that adds to addresses)
    const int sub = rows > 1 ? (lane >> gs) / heads : 0, lane_head = (lane >> gs) - sub * heads;
    const long long x_sub = sub * x_row, g_sub = sub * g_row, d_sub = sub * d_row;

    float w0[V], w1[V], dw0[V], dw1[V];
    if (NORM) {
        const char *w = is_k ? g.wk : g.wq;
        C a, b;
        a.zero();
        b.zero();
        if (p.has_a) a.load(w + p.a * E);
        if (p.has_b) b.load(w + p.b * E);
        a.widen(w0);
        b.widen(w1);
#pragma unroll
        for (int e = 0; e < V; ++e) dw0[e] = dw1[e] = 0.f;
    }
    for (int row = first / units, unit = first % units; row < T; row += row_step, unit += unit_step) {
        if (unit >= units) {
            unit -= units;
            if (++row >= T) break;
        }
        const bool on = unit * per + lane_head < heads && sub < rows && (rows == 1 || row * rows + sub < g.T);
        float c[V], s[V];
        if (g.s.rot) {
            const int pos = rows == 1 ? g.pos[row] : g.pos[min(row * rows + sub, g.T - 1)], at = min(max(pos, 0), g.n_pos - 1);
            load_angles<V, INTERLEAVED>(g.cos, g.sin, (size_t)at * g.s.half, p, c, s);
        }
        const long long offset = (long long)(unit * per + lane_head) * (g.s.d * E);
        const char *x_at = xs + (long long)row * rows * x_row + x_sub + offset, *g_at = gs_in + (long long)row * rows * g_row + g_sub + offset;
        char *d_at = outs + (long long)row * rows * d_row + d_sub + offset;
        C xa, xb, ga, gb;
        xa.zero(); xb.zero(); ga.zero(); gb.zero();
        if (on && p.has_a) {
            ga.load(g_at + p.a * E);
            if (NORM) xa.load(x_at + p.a * E);
        }
        if (on && p.has_b) {
            gb.load(g_at + p.b * E);
            if (NORM) xb.load(x_at + p.b * E);
        }
        float u[V], v[V];
        ga.widen(u);
        gb.widen(v);
        turn<V, INTERLEAVED, true>(u, v, c, s, p);
        if (NORM) {
            float x[V], y[V], sums[2] = {0.f, 0.f};    // of x x, of x u
            xa.widen(x);
            xb.widen(y);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xe = e < p.again_a ? 0.f : x[e], ye = e < p.again_b ? 0.f : y[e];
                sums[0] = fmaf(xe, xe, sums[0]);
                sums[0] = fmaf(ye, ye, sums[0]);
                sums[1] = fmaf(u[e] * w0[e], xe, sums[1]);
                sums[1] = fmaf(v[e] * w1[e], ye, sums[1]);
            }
            head_sum<2>(sums, gs);
            // (lanes without a head would add 0 times infinity to the weights' sums where eps is 0)
            const float r = on ? rsqrtf(fmaf(sums[0], g.inv_d, g.eps)) : 0.f, m = r * (sums[1] * g.inv_d);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xr = x[e] * r, yr = y[e] * r;
                dw0[e] = fmaf(u[e], xr, dw0[e]);
                dw1[e] = fmaf(v[e], yr, dw1[e]);
                u[e] = r * (u[e] * w0[e] - xr * m);
                v[e] = r * (v[e] * w1[e] - yr * m);
            }
        }
        ga.narrow(u);
        gb.narrow(v);
        if (on && p.has_a) ga.template store<true>(d_at + p.a * E);
        if (on && p.has_b) gb.template store<true>(d_at + p.b * E);
    }
    if (NORM) {
        __shared__ float red[BACK_WAVES][256];
        sum_over_heads<V>(dw0, gs);
        sum_over_heads<V>(dw1, gs);
        if (lane < (1 << gs)) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (p.has_a) red[wave][p.a + e] = dw0[e];
                if (p.has_b) red[wave][p.b + e] = dw1[e];
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * g.s.d; i += blockDim.x) {
            const int kind = i >= g.s.d, e = i - kind * g.s.d;
            float sum = 0.f;
            for (int w = kind ? g.wq_waves : 0; w < (kind ? waves : g.wq_waves); ++w) sum += red[w][e];
            if (gridDim.x == 1) (kind ? g.dwk : g.dwq)[e] = sum;
            else g.partial[(size_t)blockIdx.x * 2 * g.s.d + i] = sum;
        }
    }
}

// dw[i] = the workgroups' partial sums added in a fixed order; 16 columns a workgroup, 64 threads a column.
__global__ __launch_bounds__(1024) void heads_weights_kernel(const float *__restrict__ partial, int parts, int d, float *__restrict__ dwq,
                                                             float *__restrict__ dwk)
{
    __shared__ float red[64][17];
    const int col = threadIdx.x & 15, sl = threadIdx.x >> 4, i = blockIdx.x * 16 + col;
    float x[4], sum = 0.f;
    for (int first = sl; first < parts; first += 256) {      // (once: there are at most 256 workgroups)
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = i < 2 * d && first + 64 * u < parts ? partial[(size_t)(first + 64 * u) * 2 * d + i] : 0.f;
        sum += (x[0] + x[1]) + (x[2] + x[3]);
    }
    red[sl][col] = sum;
    __syncthreads();
    float v[1] = {red[threadIdx.x & 63][threadIdx.x >> 6]};      // a column's sums on the lanes of a wavefront
    head_sum<1>(v, 6);
    const int o = blockIdx.x * 16 + (threadIdx.x >> 6);
    if ((threadIdx.x & 63) == 0 && o < 2 * d) (o < d ? dwq[o] : dwk[o - d]) = v[0];
}

struct TableSpec {
    double exponent;        // theta_i = 2^(i exponent)
    double shrink;          // 1 / factor; 1 where nothing is scaled
    double slope, start;    // what is kept of theta_i: turns of a position * slope + start, between 0 and 1
    double magnitude;
    int mix;                // scaled by parts
};

// Cosines and sines.  A thread keeps to one pair and steps through the rows: angles are added by multiplying exp(i angle) by exp(i step) in 64
// bits, so that sines themselves are computed twice a thread.
__global__ __launch_bounds__(256) void rope_tables_kernel(float *__restrict__ cos, float *__restrict__ sin, long long first, long long rows,
                                                          int half, int steps, TableSpec spec)
{
    const int at_once = 256 / half;      // rows of a pass
    const int i = threadIdx.x % half, sub = threadIdx.x / half;
    if (sub >= at_once) return;
    double turns = exp2(i * spec.exponent) * 0.159154943091895335768884;     // of a position: theta_i / 2 pi
    const double keep = spec.mix ? fmin(fmax(turns * spec.slope + spec.start, 0.0), 1.0) : 0.0;
    turns *= keep + (1.0 - keep) * spec.shrink;
    long long row = (long long)blockIdx.x * at_once * steps + sub;
    double t = (double)(first + row) * turns, c, s, dc = 1.0, ds = 0.0;
    sincospi(2.0 * (t - rint(t)), &s, &c);
    if (steps > 1) {
        t = at_once * turns;
        sincospi(2.0 * (t - rint(t)), &ds, &dc);
    }
    c *= spec.magnitude;
    s *= spec.magnitude;
    for (int k = 0; k < steps && row < rows; ++k, row += at_once) {
        cos[row * half + i] = (float)c;
        sin[row * half + i] = (float)s;
        const double n = c * dc - s * ds;
        s = s * dc + c * ds;
        c = n;
    }
}

// ---- host ---------------------------------------------------------------------------------------
static inline bool off16(const void *p) { return ((uintptr_t)p & 15) != 0; }

static int check_heads(const alora_heads_dims *d)
{
    if (!d) return ALORA_EINVAL;
    if (d->dtype != ALORA_F32 && d->dtype != ALORA_BF16) return ALORA_EINVAL;
    if (d->n_tokens < 0 || d->n_q_heads < 1 || d->n_kv_heads < 1 || d->head_dim < 1 || d->rotary_dim < 0 || d->n_slots < 0) return ALORA_EINVAL;
    if ((d->interleaved | 1) != 1 || (d->norm | 1) != 1 || !(d->eps >= 0.f) || std::isinf(d->eps)) return ALORA_EINVAL;
    if (d->rotary_dim && d->rope_positions < 1) return ALORA_EINVAL;
    if (d->head_dim > 256 || d->head_dim % (d->dtype == ALORA_BF16 ? 8 : 4) || d->rotary_dim % 4 || d->rotary_dim > d->head_dim) return ALORA_ESHAPE;
    if (d->n_q_heads > 0x3fffffff / d->head_dim || d->n_kv_heads > 0x3fffffff / d->head_dim) return ALORA_ESHAPE;
    if ((long long)d->n_tokens * (d->n_q_heads + 2ll * d->n_kv_heads) > 0x7fffffffll) return ALORA_ESHAPE;
    return ALORA_OK;
}

// a stride that holds the row and keeps 16-byte alignment
static bool bad_stride(int64_t stride, int64_t width, int dtype) { return stride < width || stride % (dtype == ALORA_BF16 ? 8 : 4) || stride > (1ll << 40); }

// V and the layout as template arguments: f(integral_constant V, bool_constant bf16, bool_constant interleaved)
template <typename F>
static int with_layout(bool bf16, int V, bool interleaved, F f)
{
    using std::integral_constant;
    using std::bool_constant;
#define ALORA_CASE(B, N, I) \
    if (bf16 == B && V == N && interleaved == I) return f(bool_constant<B>(), integral_constant<int, N>(), bool_constant<I>());
    ALORA_CASE(true, 8, false)
    ALORA_CASE(true, 4, false)
    ALORA_CASE(true, 2, false)
    ALORA_CASE(true, 8, true)
    ALORA_CASE(true, 4, true)
    ALORA_CASE(false, 4, false)
    ALORA_CASE(false, 2, false)
    ALORA_CASE(false, 4, true)
#undef ALORA_CASE
    return -1;
}

static int units_of(int heads, const HeadShape &s)
{
    const int per = 64 >> s.gshift;
    return (heads + per - 1) / per;
}

static int launch_heads(HeadsArgs &g, bool bf16, int V, bool norm, hipStream_t st)
{
    const uint32_t v_bytes = g.v ? (uint32_t)g.hkv * g.s.d * (bf16 ? 2 : 4) : 0u;
    const int units = g.uq + g.uk, v_pieces = pieces_of(v_bytes);
    // Units of a wavefront: one where the chip is not full many times over (more wavefronts have shorter chains of loads), else three where
    // that comes out even, else two.  us with two | three: 9 units, 8192 rows 71.8 | 61.6, 6 units, 4096 rows 27.2 | 25.4; 8 units, 4096 rows
    // 40.3 | 43.6, 10 units 39.5 | 40.9, 5 units 18.9 | 19.1, 2048 rows 11.4 | 12.1.  Four: 67.4, 28.4, 49.6, 42.5, 20.7, 13.4.
    const int U = (long long)g.T * units < 8192 ? 1 : units % 3 ? 2 : 3;
    const int per = 64 >> g.s.gshift;
    const auto items = [&](int at_once) { return (g.T + at_once - 1) / std::max(1, at_once); };
    g.items_q = items(per / g.hq);
    g.items_k = items(per / g.hkv);
    const long long all = (long long)g.items_q + g.items_k + (g.v ? items(128 / (int)(v_bytes / 16)) : 0);
    if (g.hq <= per / 2 && g.hkv <= per / 2 && all <= (1 << 26) - 4) {     // (a grid holds fewer than 2^32 threads: 2^24 - 1 workgroups of 256)
        return with_layout(bf16, V, g.s.interleaved, [&](auto b, auto v, auto il) {
            const auto go = [&](auto kernel) {
                launch_kernel(kernel, dim3((unsigned)((all + 3) / 4)), dim3(256), 0, st, g);
                return launch_status();
            };
            return norm ? go(heads_packed_kernel<b.value, v.value, il.value, true>) : go(heads_packed_kernel<b.value, v.value, il.value, false>);
        });
    }
    const int waves = std::min(HEADS_WAVES, (units + U - 1) / U + v_pieces);
    return with_layout(bf16, V, g.s.interleaved, [&](auto b, auto v, auto il) {
        const auto go = [&](auto kernel) {
            launch_kernel(kernel, dim3(std::min(g.T, ROWS_AT_ONCE), (g.T - 1) / ROWS_AT_ONCE + 1), dim3(64 * waves), 0, st, g);
            return launch_status();
        };
        const auto with = [&](auto n) {
            return U == 3 ? go(heads_kernel<b.value, v.value, il.value, n.value, 3>)
                          : U == 2 ? go(heads_kernel<b.value, v.value, il.value, n.value, 2>) : go(heads_kernel<b.value, v.value, il.value, n.value, 1>);
        };
        return norm ? with(std::true_type()) : with(std::false_type());
    });
}

// Workgroups of the backward pass, each with a row of partial sums.
struct BackPlan {
    int groups, waves, q_waves;   // workgroups, their wavefronts, those of them that take queries
};
// Units that one workgroup takes alone, without the second kernel; the pass in us with it and without: 5 units 11.2 and 8.4, 40 units 11.1 and
// 9.5, 80 units 11.1 and 13.9.
constexpr int ONE_WORKGROUP = 48;
// rows of `heads` heads that share a unit
static int rows_of(int heads, const HeadShape &s) { return std::max(1, (64 >> s.gshift) / heads); }

// Eight wavefronts a workgroup where the units are few, so that fewer partial sums are left; the first kernel in us with 2 | 4 | 8 | 16: 613 fp32 rows of 4 / 2
// heads of 64 5.4 | 4.8 | 4.9 | 6.0, 128 rows of 32 / 8 heads of 128 6.6 | 6.6 | 6.0 | 7.3.
static BackPlan plan_back(int T, int hq, int hkv, const HeadShape &s)
{
    const auto units = [&](int heads) { return (T + rows_of(heads, s) - 1) / rows_of(heads, s) * (long long)units_of(heads, s); };
    const long long uq = units(hq), uk = units(hkv), all = uq + uk;
    const int most = all <= ONE_WORKGROUP ? BACK_WAVES : (int)std::min<long long>(BACK_WAVES, std::max<long long>(8, all / 256));
    BackPlan p = {0, 0, 0};
    if (T == 0) return p;
    double best = 0.0;
    for (int w = 2; w <= most; ++w) {
        const int q = std::max(1, std::min(w - 1, (int)((double)w * uq / (uq + uk) + 0.5)));
        const double cost = std::max((double)uq / q, (double)uk / (w - q)) * w;    // wavefronts' time
        if (w == 2 || cost <= best * 1.02) {
            best = w == 2 ? cost : std::min(best, cost);
            p.waves = w;
            p.q_waves = q;
        }
    }
    p.groups = all <= ONE_WORKGROUP ? 1 : (int)std::min<long long>(256, (all + p.waves - 1) / p.waves);
    return p;
}

static HeadShape shape_of(const alora_heads_dims *d) { return head_shape(d->head_dim, d->rotary_dim, d->interleaved, head_chunk(d->dtype == ALORA_BF16, d->head_dim, d->rotary_dim, d->interleaved)); }

static size_t back_workspace(const alora_heads_dims *d)
{
    const HeadShape s = shape_of(d);
    const int groups = plan_back(d->n_tokens, d->n_q_heads, d->n_kv_heads, s).groups;
    return d->norm && groups > 1 ? (size_t)groups * 2 * d->head_dim * sizeof(float) : 0;
}

}  // namespace alora

using namespace alora;

extern "C" {

int alora_qk_norm_rope(const void *q, void *q_out, const void *k, void *k_cache, const void *v, void *v_cache, const void *wq, const void *wk,
                       const float *cos, const float *sin, const int32_t *positions, const int64_t *slot_mapping, const alora_heads_dims *dims,
                       void *hip_stream)
{
    const int st = check_heads(dims);
    if (st) return st;
    const alora_heads_dims &d = *dims;
    if (d.n_tokens == 0) return ALORA_OK;
    const int64_t Nq = (int64_t)d.n_q_heads * d.head_dim, Nkv = (int64_t)d.n_kv_heads * d.head_dim;
    if (!q || !q_out || !slot_mapping || (d.n_slots && !k_cache)) return ALORA_EINVAL;
    if (!v != !v_cache && d.n_slots) return ALORA_EINVAL;
    if ((wq != nullptr) != (d.norm != 0) || (wk != nullptr) != (d.norm != 0)) return ALORA_EINVAL;
    if ((cos != nullptr) != (d.rotary_dim > 0) || (sin != nullptr) != (d.rotary_dim > 0) || (d.rotary_dim && !positions)) return ALORA_EINVAL;
    if (off16(q) || off16(q_out) || off16(k) || off16(k_cache) || off16(v) || off16(v_cache) || off16(wq) || off16(wk) || off16(cos) || off16(sin) ||
        ((uintptr_t)positions & 3) || ((uintptr_t)slot_mapping & 7))
        return ALORA_EINVAL;
    if (bad_stride(d.q_stride, Nq, d.dtype) || bad_stride(d.q_out_stride, Nq, d.dtype) || bad_stride(d.k_out_stride, Nkv, d.dtype) ||
        (k && bad_stride(d.k_stride, Nkv, d.dtype)) || (v && (bad_stride(d.v_stride, Nkv, d.dtype) || bad_stride(d.v_out_stride, Nkv, d.dtype))) ||
        (q == q_out && d.q_stride != d.q_out_stride))
        return ALORA_EINVAL;
    const bool bf16 = d.dtype == ALORA_BF16;
    const int E = bf16 ? 2 : 4, V = head_chunk(bf16, d.head_dim, d.rotary_dim, d.interleaved);
    HeadsArgs g;
    g.q = (const char *)q; g.q_out = (char *)q_out; g.k = (const char *)k; g.kc = (char *)k_cache;
    g.v = (const char *)v; g.vc = (char *)v_cache; g.wq = (const char *)wq; g.wk = (const char *)wk;
    g.cos = cos; g.sin = sin; g.pos = positions; g.slot = slot_mapping;
    g.q_row = d.q_stride * E; g.qo_row = d.q_out_stride * E; g.k_row = d.k_stride * E; g.ko_row = d.k_out_stride * E;
    g.v_row = d.v_stride * E; g.vo_row = d.v_out_stride * E;
    g.n_slots = d.n_slots;
    g.s = head_shape(d.head_dim, d.rotary_dim, d.interleaved, V);
    g.T = d.n_tokens; g.hq = d.n_q_heads; g.hkv = d.n_kv_heads; g.n_pos = d.rope_positions;
    g.uq = units_of(g.hq, g.s); g.uk = units_of(g.hkv, g.s);
    g.eps = d.eps; g.inv_d = 1.0f / (float)d.head_dim;
    const int e = launch_heads(g, bf16, V, d.norm, (hipStream_t)hip_stream);
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

int alora_qk_norm_rope_workspace_bytes(const alora_heads_dims *dims, size_t *out_bytes)
{
    if (!out_bytes) return ALORA_EINVAL;
    const int st = check_heads(dims);
    if (st) return st;
    *out_bytes = back_workspace(dims);
    return ALORA_OK;
}

int alora_qk_norm_rope_backward(const void *q, const void *dq_out, void *dq, const void *k, const void *dk_out, void *dk, const void *wq,
                                const void *wk, float *dwq, float *dwk, const float *cos, const float *sin, const int32_t *positions,
                                const alora_heads_dims *dims, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int st = check_heads(dims);
    if (st) return st;
    const alora_heads_dims &d = *dims;
    const int64_t Nq = (int64_t)d.n_q_heads * d.head_dim, Nkv = (int64_t)d.n_kv_heads * d.head_dim;
    if ((wq != nullptr) != (d.norm != 0) || (wk != nullptr) != (d.norm != 0) || (dwq != nullptr) != (d.norm != 0) || (dwk != nullptr) != (d.norm != 0))
        return ALORA_EINVAL;
    if (off16(wq) || off16(wk) || off16(dwq) || off16(dwk)) return ALORA_EINVAL;
    const int64_t dq_stride = d.dq_stride ? d.dq_stride : d.q_stride, dk_stride = d.dk_stride ? d.dk_stride : d.k_stride;
    if (d.n_tokens) {
        if (!q || !dq_out || !dq || !k || !dk_out || !dk) return ALORA_EINVAL;
        if ((cos != nullptr) != (d.rotary_dim > 0) || (sin != nullptr) != (d.rotary_dim > 0) || (d.rotary_dim && !positions)) return ALORA_EINVAL;
        if (off16(q) || off16(dq_out) || off16(dq) || off16(k) || off16(dk_out) || off16(dk) || off16(cos) || off16(sin) || ((uintptr_t)positions & 3))
            return ALORA_EINVAL;
        if (bad_stride(d.q_stride, Nq, d.dtype) || bad_stride(d.q_out_stride, Nq, d.dtype) || bad_stride(d.k_stride, Nkv, d.dtype) ||
            bad_stride(d.k_out_stride, Nkv, d.dtype) || bad_stride(dq_stride, Nq, d.dtype) || bad_stride(dk_stride, Nkv, d.dtype) ||
            (dq == dq_out && dq_stride != d.q_out_stride) || (dk == dk_out && dk_stride != d.k_out_stride))
            return ALORA_EINVAL;
    }
    const size_t need = back_workspace(dims);
    if (need && (!workspace || off16(workspace) || workspace_bytes < need)) return ALORA_EWORKSPACE;
    const bool bf16 = d.dtype == ALORA_BF16;
    const int E = bf16 ? 2 : 4, V = head_chunk(bf16, d.head_dim, d.rotary_dim, d.interleaved);
    HeadsBackArgs g;
    g.q = (const char *)q; g.k = (const char *)k; g.gq = (const char *)dq_out; g.gk = (const char *)dk_out; g.dq = (char *)dq; g.dk = (char *)dk;
    g.wq = (const char *)wq; g.wk = (const char *)wk;
    g.cos = cos; g.sin = sin; g.pos = positions;
    g.q_row = d.q_stride * E; g.k_row = d.k_stride * E; g.gq_row = d.q_out_stride * E; g.gk_row = d.k_out_stride * E;
    g.dq_row = dq_stride * E; g.dk_row = dk_stride * E;
    g.partial = (float *)workspace;
    g.s = head_shape(d.head_dim, d.rotary_dim, d.interleaved, V);
    g.T = d.n_tokens; g.hq = d.n_q_heads; g.hkv = d.n_kv_heads; g.n_pos = d.rope_positions;
    g.uq = units_of(g.hq, g.s); g.uk = units_of(g.hkv, g.s);
    g.eps = d.eps; g.inv_d = 1.0f / (float)d.head_dim;
    g.rows_q = rows_of(g.hq, g.s); g.rows_k = rows_of(g.hkv, g.s);
    const BackPlan plan = plan_back(d.n_tokens, g.hq, g.hkv, g.s);
    g.wq_waves = plan.q_waves;
    g.dwq = dwq; g.dwk = dwk;
    const hipStream_t stream = (hipStream_t)hip_stream;
    int e = 0;
    if (plan.groups)
        e = with_layout(bf16, V, d.interleaved, [&](auto b, auto v, auto il) {
            if (d.norm) launch_kernel(heads_back_kernel<b.value, v.value, il.value, true>, dim3(plan.groups), dim3(64 * plan.waves), 0, stream, g);
            else launch_kernel(heads_back_kernel<b.value, v.value, il.value, false>, dim3(plan.groups), dim3(64 * plan.waves), 0, stream, g);
            return launch_status();
        });
    if (!e && d.norm && plan.groups != 1) {
        launch_kernel(heads_weights_kernel, dim3((2 * d.head_dim + 15) / 16), dim3(1024), 0, stream, (const float *)workspace, plan.groups, (int)d.head_dim, dwq, dwk);
        e = launch_status();
    }
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

int alora_qk_norm_rope_validate(const int32_t *positions, const int64_t *slot_mapping, const alora_heads_dims *dims)
{
    const int st = check_heads(dims);
    if (st) return st;
    const size_t T = (size_t)dims->n_tokens;
    if (T == 0) return ALORA_OK;
    if (!slot_mapping || (dims->rotary_dim && !positions)) return ALORA_EINVAL;
    try {
        std::vector<int32_t> pos(dims->rotary_dim ? T : 0);
        std::vector<int64_t> slot(T);
        hipError_t e = hipMemcpy(slot.data(), slot_mapping, 8 * T, hipMemcpyDeviceToHost);
        if (!e && dims->rotary_dim) e = hipMemcpy(pos.data(), positions, 4 * T, hipMemcpyDeviceToHost);
        if (e) { note_hip_error((int)e); return ALORA_EHIP; }
        for (int32_t x : pos)
            if (x < 0 || x >= dims->rope_positions) return ALORA_EDATA;
        std::sort(slot.begin(), slot.end());
        if (slot.front() < -1 || slot.back() >= dims->n_slots) return ALORA_EDATA;
        for (size_t i = 1; i < T; ++i)
            if (slot[i] >= 0 && slot[i] == slot[i - 1]) return ALORA_EDATA;
        return ALORA_OK;
    } catch (const std::bad_alloc &) {
        return ALORA_ENOMEM;
    }
}

int alora_rope_tables(float *cos, float *sin, int64_t first, int64_t rows, const alora_rope_spec *spec, void *hip_stream)
{
    if (!spec || first < 0 || rows < 0) return ALORA_EINVAL;
    const alora_rope_spec &s = *spec;
    if (s.scaling < ALORA_ROPE_PLAIN || s.scaling > ALORA_ROPE_BY_PARTS || !(s.base > 0.0) || std::isinf(s.base) || !std::isfinite(s.magnitude)) return ALORA_EINVAL;
    if (s.scaling != ALORA_ROPE_PLAIN && (!(s.factor > 0.0) || std::isinf(s.factor))) return ALORA_EINVAL;
    if (s.scaling == ALORA_ROPE_BY_PARTS && (!(s.original > 0.0) || std::isinf(s.original) || !std::isfinite(s.low) || !std::isfinite(s.high) || !(s.low < s.high)))
        return ALORA_EINVAL;
    if (s.rotary_dim < 2 || s.rotary_dim > 512 || s.rotary_dim % 2) return ALORA_ESHAPE;
    if (first > (1 << 24) || rows > (1 << 24) - first) return ALORA_ESHAPE;
    if (rows == 0) return ALORA_OK;
    if (!cos || !sin || off16(cos) || off16(sin)) return ALORA_EINVAL;
    const int half = s.rotary_dim / 2, at_once = 256 / half;
    // rows per thread: about 512 workgroups, at most 64 steps.  us with 512 | 1024 | 2048 workgroups, 64 pairs: 16384 rows 6.2 | 6.5 | 8.2,
    // 65536 rows 8.8 | 9.1 | 10.8, 131072 rows 13.3 | 13.2 | 13.2; two or four pairs a thread with wider stores: 6.4 to 22
    const int steps = (int)std::max<int64_t>(1, std::min<int64_t>(64, rows / ((int64_t)at_once * 512)));
    const int64_t groups = (rows + (int64_t)at_once * steps - 1) / ((int64_t)at_once * steps);
    TableSpec t = {-std::log2(s.base) / half, s.scaling == ALORA_ROPE_PLAIN ? 1.0 : 1.0 / s.factor, 0.0, 0.0, s.magnitude, s.scaling == ALORA_ROPE_BY_PARTS};
    if (t.mix) {
        t.slope = s.original / (s.high - s.low);
        t.start = -s.low / (s.high - s.low);
    }
    launch_kernel(rope_tables_kernel, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)hip_stream, cos, sin, (long long)first, (long long)rows, half, steps, t);
    const int e = launch_status();
    if (e) { note_hip_error(e); return ALORA_EHIP; }
    return ALORA_OK;
}

}  // extern "C"
