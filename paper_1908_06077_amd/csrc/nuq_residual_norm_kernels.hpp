// The seam between two blocks of a transformer, forward and backward: a norm of the branch, gate, dropout, scales and the residual
// sum, and the norm of the sum.
//
//   n = N1(x), n' = n w1 + b1 (or x);  t = residual_scale residual + scale gate drop(n'), rounded to x's type;  y = N2(t) w2 + b2
//   N(s) = (s - mean) rstd, rstd = 1 / sqrt(mean((s - mean)^2) + eps); the root-mean-square norm takes 0 for the mean
//
//   with n2 = N2(t), d = dy w2:  dt = dtotal + rstd2 (d - mean(d) - n2 mean(d n2));  dw2 = sum dy n2;  db2 = sum dy
//   dresidual = residual_scale dt;  g = scale drop(dt);  dgate = sum g n';  h = g gate;  dw1 = sum h n;  db1 = sum h
//   dx = rstd1 (h w1 - mean(h w1) - n mean(h w1 n))      (mean(.) alone falls away in the root-mean-square norm; sums are over rows)
//
// The five sums over rows are four: with u = drop(dt) / keep and c = scale keep, U1 = sum u n and U0 = sum u,
//   dw1 = c gate U1;  db1 = c gate U0;  dgate = c (w1 U1 + b1 U0);  and h w1 = u (c gate w1)
// A row stays in the registers of one team of threads from its loads to its results: two rows are read and two written forward,
// four read and two written backward, whatever is fused.  Statistics and sums are fp32, the variance is taken of centred values,
// results are rounded to their type once.  The mask is computed again in the backward pass.  Bound by HBM, and on short batches by
// latency.  kOnce: rows that together do not fit the last-level cache are read and written with that hint (16384 x 8192 in bfloat16
// backward 307 -> 281 us).
// Measured, both norms, gate, bias and dropout, bfloat16: 8192 rows of 1600 forward 27 us (3.9 TB/s of 105 MB), backward 38 us (4.1 of
// 157 MB) and 6.5 us for the launch that adds the sums up.  There neither HBM nor the vector units are the bound by themselves: these issue
// in 0.66 (forward, 44 instructions per element) and 0.73 (backward, 68) of the cycles, and waves wait in half of theirs, for memory and at
// the barriers of a row, which a CU's only workgroup of 1024 threads (backward: two of 512) meets at.  16384 of 8192 backward, root-mean-square norms, 266 us (6.1 TB/s) and 12.
#pragma once

#include <type_traits>

#include "nuq_dropout_kernels.hpp"

namespace nuq {

enum NormKind : uint32_t { kNoNorm = NUQ_NO_NORM, kLayerNorm = NUQ_LAYER_NORM, kRmsNorm = NUQ_RMS_NORM };

struct ResidualNormForward {
    const void *x, *residual;                  // residual: may be none
    const void *w1, *b1, *gate, *w2, *b2;      // each may be none
    void *total, *y;                           // y: where there is an outer norm
    float *stats;                              // [4][rows]: mean1, rstd1, mean2, rstd2; may be none
    Draws draws;
    uint64_t rows, ldx, ldr, ldt, ldy;
    uint32_t hidden, inner, outer;
    float eps, factor, residual_scale;         // factor: scale times what is kept is multiplied with
};

// Sums over the threads of a row, one after the other, the same bits in each: a set of red is not written again before a barrier that
// follows its last read, because the two sets take turns.  The teams of a workgroup meet at the barriers of teams of several waves.
template <int TEAM, int WAVES>
struct RowSums {
    float (&red)[2][WAVES];
    uint32_t turn;
    __device__ __forceinline__ float operator()(float x)
    {
        if constexpr (TEAM <= 64) {
            return team_sum<TEAM>(x);
        } else {
            turn ^= 1u;
            x = team_sum<64>(x);
            if (threadIdx.x % 64u == 0)
                red[turn][threadIdx.x / 64u] = x;
            __syncthreads();
            const uint32_t own = threadIdx.x / TEAM * (TEAM / 64);
            x = red[turn][own];
#pragma unroll
            for (int k = 1; k < TEAM / 64; ++k)
                x += red[turn][own + k];
            return x;
        }
    }
};

// Loads that are not part of a sum have arrived here: what follows the next barrier may be stored where another thread read.
template <class V, int NV>
__device__ __forceinline__ void arrived(const V (&x)[NV])
{
#pragma unroll
    for (int k = 0; k < NV; ++k)
        asm volatile("" ::"v"(x[k]));
}

// add(k, e) for the elements of a row that count, which are not a neighbour's too: `whole`, where the row is whole vectors, as one choice
// per vector.  The two numbers that add() adds to.
struct Pair {
    float a, b;
};
template <class Shape, int NV, int VEC, class F>
__device__ __forceinline__ Pair add_up(const Shape &S, bool whole, F &&add)
{
    Pair all{0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        Pair part = all;
        if (whole) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                add(k, e, part);
            all = S.there(k) ? part : all;
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                Pair next = all;
                add(k, e, next);
                all = S.counts(k, e) ? next : all;
            }
        }
    }
    return all;
}

// s <- N(s), its mean and reciprocal deviation.  between(): behind the first barrier, before s changes.
template <class Sums, class Shape, int NV, int VEC, class F>
__device__ __forceinline__ void norm_row(float (&s)[NV][VEC], const Shape &S, bool whole, Sums &sums, uint32_t kind, float per, float eps,
                                         float &mean, float &rstd, F &&between)
{
    mean = 0.0f;
    if (kind == kLayerNorm) {
        mean = sums(add_up<Shape, NV, VEC>(S, whole, [&](int k, int e, Pair &p) { p.a += s[k][e]; }).a) * per;
        between();
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s[k][e] -= mean;
    }
    const float square = sums(add_up<Shape, NV, VEC>(S, whole, [&](int k, int e, Pair &p) { p.a = __builtin_fmaf(s[k][e], s[k][e], p.a); }).a);
    rstd = 1.0f / __builtin_sqrtf(square * per + eps);
    if (kind != kLayerNorm)
        between();
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            s[k][e] *= rstd;
}

// Vectors of `hidden` floats in the LDS for all teams of a workgroup, as the team's threads have the row: written by its first team, read
// by the thread of a team that has the same columns.  Registers are what waves per SIMD depend on, and those the bytes on their way.
template <int COUNT, class Shape>
struct TeamVectors {
    static constexpr int UNIT = Shape::VEC < 4 ? Shape::VEC : 4, UNITS = Shape::NV * Shape::VEC / UNIT;
    typedef float Unit __attribute__((ext_vector_type(UNIT)));
    using Memory = Unit[COUNT][UNITS][Shape::TEAM];
    Memory &at;
    __device__ __forceinline__ void put(int which, const float (&x)[Shape::NV][Shape::VEC])
    {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            Unit v;
#pragma unroll
            for (int e = 0; e < UNIT; ++e)
                v[e] = x[(u * UNIT + e) / Shape::VEC][(u * UNIT + e) % Shape::VEC];
            at[which][u][threadIdx.x % (uint32_t)Shape::TEAM] = v;
        }
    }
    __device__ __forceinline__ void get(int which, float (&x)[Shape::NV][Shape::VEC]) const
    {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const Unit v = at[which][u][threadIdx.x % (uint32_t)Shape::TEAM];
#pragma unroll
            for (int e = 0; e < UNIT; ++e)
                x[(u * UNIT + e) / Shape::VEC][(u * UNIT + e) % Shape::VEC] = v[e];
        }
    }
};

// to[k][e] <- the vector's element of that place, or `other` where there is no vector.
template <class W, class Shape, int NV, int VEC>
__device__ __forceinline__ void vector_or(float (&to)[NV][VEC], const void *from, const Shape &S, float other)
{
    Vec<W, VEC> x[NV];
    if (from)
        S.load(x, static_cast<const W *>(from));
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            to[k][e] = from ? (float)x[k][e] : other;
}

// A vector of weights where a team has few rows: in its registers (kHold), or read where it is used.
template <class Shape, class W, int NV, int VEC, bool kHold>
struct RowVector {
    const W *from;
    Vec<W, VEC> held[kHold ? NV : 1];
    __device__ __forceinline__ RowVector(const void *p, const Shape &S) : from(static_cast<const W *>(p))
    {
        if constexpr (kHold)
            if (from)
                S.load(held, from);
    }
    // f(k, e, weight) for the row's elements, where there is a vector.
    template <class F>
    __device__ __forceinline__ void apply(const Shape &S, F &&f) const
    {
        if (!from)
            return;
        if constexpr (kHold) {
            each(held, f);
        } else {
            Vec<W, VEC> now[NV];
            S.load(now, from);
            each(now, f);
        }
    }

private:
    template <class F>
    static __device__ __forceinline__ void each(const Vec<W, VEC> (&w)[NV], F &&f)
    {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                f(k, e, (float)w[k][e]);
    }
};

// Forward: threads of a workgroup.  kMany: there are many rows per team.  What is done to n1 and n2 is then one multiply-add each, by
// vectors in the LDS: A = w1 gate factor, B = b1 gate factor, w2, b2.
template <int TEAM, bool kMany>
constexpr int kSeamForwardWG = kMany ? 1024 : TEAM <= 64 ? 256 : TEAM;

template <class T, class W, int TEAM, int E, int VEC, bool kInner, bool kMany, bool kOnce>
__global__ __launch_bounds__((kSeamForwardWG<TEAM, kMany>)) void k_residual_norm_forward(const ResidualNormForward P)
{
    using Shape = RowShape<T, TEAM, E, VEC>;
    constexpr int NV = Shape::NV, WG = kSeamForwardWG<TEAM, kMany>, TEAMS = WG / TEAM;
    constexpr bool kAhead = kMany || E <= 8;                 // (the next row in registers: not beside sixteen elements and their weights)
    using Few = RowVector<Shape, W, NV, VEC, (!kMany && E <= 8)>;
    using Many = TeamVectors<4, Shape>;
    __shared__ typename std::conditional<kMany, typename Many::Memory, char>::type kept;
    __shared__ float red[2][WG / 64];
    const uint32_t hidden = P.hidden;
    const bool whole = hidden % VEC == 0;
    const float per = 1.0f / (float)hidden;
    const Shape S(hidden);
    RowSums<TEAM, WG / 64> sums{red, 0u};
    uint32_t team = threadIdx.x / TEAM;
    if constexpr (TEAM >= 64)
        team = uniform_u32(team);
    const uint64_t begin = P.draws.begin();
    Vec<T, VEC> xs[NV], rs[NV];
    const T *const residual = static_cast<const T *>(P.residual ? P.residual : P.x);        // (without one, x: read, and not used)
    const uint64_t ldr = P.residual ? P.ldr : P.ldx;
    // (a team without a row in the workgroup's last turn takes the last row along, and writes nothing: teams meet at barriers)
    const auto row_of = [&](uint64_t first) { return min(first + team, P.rows - 1u); };
    const uint64_t turn = (uint64_t)gridDim.x * TEAMS;
    uint64_t first = (uint64_t)blockIdx.x * TEAMS;
    if constexpr (kAhead) {
        S.template load<kOnce>(xs, static_cast<const T *>(P.x) + row_of(first) * P.ldx);
        S.template load<kOnce>(rs, residual + row_of(first) * ldr);
    }
    const Few w1(kMany || !kInner ? nullptr : P.w1, S), b1(kMany || !kInner ? nullptr : P.b1, S), gate(kMany ? nullptr : P.gate, S),
        w2(kMany ? nullptr : P.w2, S), b2(kMany ? nullptr : P.b2, S);
    if constexpr (kMany) {
        Many M{kept};
        if (threadIdx.x < (uint32_t)TEAM) {
            float a[NV][VEC], b[NV][VEC], g[NV][VEC];
            vector_or<W>(g, P.gate, S, 1.0f);
            vector_or<W>(a, P.w1, S, 1.0f);
            vector_or<W>(b, P.b1, S, 0.0f);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    g[k][e] *= P.factor;
                    a[k][e] *= g[k][e];
                    b[k][e] *= g[k][e];
                }
            M.put(0, a);
            M.put(1, b);
            vector_or<W>(a, P.w2, S, 1.0f);
            vector_or<W>(b, P.b2, S, 0.0f);
            M.put(2, a);
            M.put(3, b);
        }
        __syncthreads();
    }
    for (;;) {
        const uint64_t now = row_of(first);
        const bool own = first + team < P.rows;
        if constexpr (!kAhead) {
            S.template load<kOnce>(xs, static_cast<const T *>(P.x) + now * P.ldx);
            S.template load<kOnce>(rs, residual + now * ldr);
        }
        float s[NV][VEC], mean, rstd;
        if constexpr (TEAM > 64)
            arrived(rs);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s[k][e] = (float)xs[k][e];
        first += turn;
        const bool more = first < P.rows;
        if (kAhead && more)
            S.template load<kOnce>(xs, static_cast<const T *>(P.x) + row_of(first) * P.ldx);
        if constexpr (kInner) {
            norm_row(s, S, whole, sums, P.inner, per, P.eps, mean, rstd, [] {});
            if (P.stats && own && threadIdx.x % TEAM == 0) {
                if (P.inner == kLayerNorm)
                    P.stats[now] = mean;
                P.stats[P.rows + now] = rstd;
            }
        }
        if constexpr (kMany) {
            float a[NV][VEC], b[NV][VEC];
            const Many M{kept};
            M.get(0, a);
            if constexpr (kInner)
                M.get(1, b);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    s[k][e] = kInner ? __builtin_fmaf(s[k][e], a[k][e], b[k][e]) : s[k][e] * a[k][e];
        } else {
            w1.apply(S, [&](int k, int e, float w) { s[k][e] *= w; });
            b1.apply(S, [&](int k, int e, float w) { s[k][e] += w; });
            gate.apply(S, [&](int k, int e, float w) { s[k][e] *= w; });
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    s[k][e] *= P.factor;
        }
        if (P.draws.threshold) {
            const BucketKey key = bucket_key(begin, now);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                drop<VEC>(s[k], key, S.at[k], P.draws.threshold);
        }
        if (P.residual)
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    s[k][e] = __builtin_fmaf((float)rs[k][e], P.residual_scale, s[k][e]);
        if (kAhead && more)
            S.template load<kOnce>(rs, residual + row_of(first) * ldr);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s[k][e] = (float)(T)s[k][e];
        if (P.outer == kNoNorm) {                            // (behind a barrier of the inner norm: total may be x or residual)
            if (own)
                S.template store<kOnce>(static_cast<T *>(P.total) + now * P.ldt, s);
        } else {
            norm_row(s, S, whole, sums, P.outer, per, P.eps, mean, rstd, [&] {
                if (own)
                    S.template store<kOnce>(static_cast<T *>(P.total) + now * P.ldt, s);
            });
            if (P.stats && own && threadIdx.x % TEAM == 0) {
                if (P.outer == kLayerNorm)
                    P.stats[2u * P.rows + now] = mean;
                P.stats[3u * P.rows + now] = rstd;
            }
            if constexpr (kMany) {
                float a[NV][VEC], b[NV][VEC];
                const Many M{kept};
                M.get(2, a);
                M.get(3, b);
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        s[k][e] = __builtin_fmaf(s[k][e], a[k][e], b[k][e]);
            } else {
                w2.apply(S, [&](int k, int e, float w) { s[k][e] *= w; });
                b2.apply(S, [&](int k, int e, float w) { s[k][e] += w; });
            }
            if (own)
                S.template store<kOnce>(static_cast<T *>(P.y) + now * P.ldy, s);
        }
        if (!more)
            break;
    }
}

struct ResidualNormBackward {
    const void *dy, *dtotal, *x, *total;       // dy, total: where there is an outer norm; dtotal: may be none
    const void *w1, *b1, *gate, *w2;           // each may be none
    const float *stats;
    void *dx, *dresidual;                      // dresidual: may be none
    float *partial;                            // [parts][4][hidden]: sums of u n, of u, of dy n2, of dy; or none
    float *means;                              // [2][rows] or none: mean(d), mean(d n2), for the sums that a launch of its own takes
    Draws draws;
    uint64_t rows, ldg, lda, ldx, ldt, ldd, lde;
    uint32_t hidden, inner, outer;
    float factor, residual_scale;              // factor: scale times what is kept is multiplied with
};
constexpr uint32_t kSeamSums = 4;

// Threads of a workgroup: several teams share what is written of the sums.  And waves per SIMD that the registers have to leave room for:
// four beside eight elements per thread, two beside sixteen.
template <int TEAM>
constexpr int kSeamBackwardWG = TEAM <= 512 ? 512 : TEAM;
template <int E>
constexpr int kSeamBackwardWaves = E <= 8 ? 4 : 2;

// Two sums over the threads of a row, the same bits in each; one barrier.
template <int TEAM, int WAVES>
__device__ __forceinline__ void row_sums(float &a, float &b, float (&red)[2][2][WAVES], uint32_t &turn)
{
    if constexpr (TEAM <= 64) {
        a = team_sum<TEAM>(a);
        b = team_sum<TEAM>(b);
    } else {
        constexpr int TEAM_WAVES = TEAM / 64;
        turn ^= 1u;
        a = team_sum<64>(a);
        b = team_sum<64>(b);
        if (threadIdx.x % 64u == 0) {
            red[turn][0][threadIdx.x / 64u] = a;
            red[turn][1][threadIdx.x / 64u] = b;
        }
        __syncthreads();
        const uint32_t own = threadIdx.x / TEAM * TEAM_WAVES;
        a = red[turn][0][own];
        b = red[turn][1][own];
#pragma unroll
        for (int k = 1; k < TEAM_WAVES; ++k) {
            a += red[turn][0][own + k];
            b += red[turn][1][own + k];
        }
    }
}

// kSums: with the sums over rows, in registers; workgroup p writes partial[p], and a second launch adds those up.  w2 and c gate w1 are in
// the LDS.
template <class T, class W, int TEAM, int E, int VEC, bool kInner, bool kSums, bool kOnce>
__global__ __launch_bounds__(kSeamBackwardWG<TEAM>, kSeamBackwardWaves<E>) void k_residual_norm_backward(const ResidualNormBackward P)
{
    using Shape = RowShape<T, TEAM, E, VEC>;
    constexpr int NV = Shape::NV, WG = kSeamBackwardWG<TEAM>, TEAMS = WG / TEAM, WAVES = WG / 64;
    constexpr bool kAhead = TEAM < 1024 && sizeof(T) == 2;   // (the next row in registers, where these hold it)
    using Vectors = TeamVectors<2, Shape>;
    __shared__ typename Vectors::Memory kept;
    __shared__ float red[2][2][WAVES];
    const uint32_t hidden = P.hidden;
    const bool whole = hidden % VEC == 0;
    const Shape S(hidden);
    const float per = 1.0f / (float)hidden;
    const bool outer = P.outer != kNoNorm;
    uint32_t turn = 0, team = threadIdx.x / TEAM;
    if constexpr (TEAM >= 64)
        team = uniform_u32(team);
    const uint64_t begin = P.draws.begin();
    float total_of[kSeamSums][NV][VEC] = {};
    // What a pass does without reads something that is there in its place, and does not use it.
    const T *const dy = static_cast<const T *>(outer ? P.dy : P.x), *const total = static_cast<const T *>(outer ? P.total : P.x);
    const T *const dtotal = P.dtotal ? static_cast<const T *>(P.dtotal) : dy, *const x = static_cast<const T *>(P.x);
    const uint64_t ldg = outer ? P.ldg : P.ldx, ldt = outer ? P.ldt : P.ldx, lda = P.dtotal ? P.lda : ldg;
    Vec<T, VEC> gs[NV], ts[NV], as[NV], xs[NV];
    // (The statistics with the rows: a load behind theirs would wait for them.  What a norm does not have is read, and not used.  All in one
    // place and without a condition, so that what is waited for is counted, and not everything; a team without a row takes the last one.)
    float mean1 = 0.0f, rstd1 = 0.0f, mean2 = 0.0f, rstd2 = 0.0f;
    const auto load = [&](uint64_t row) {
        row = min(row, P.rows - 1u);
        mean1 = P.stats[row];
        rstd1 = P.stats[P.rows + row];
        mean2 = P.stats[2u * P.rows + row];
        rstd2 = P.stats[3u * P.rows + row];
        S.template load<kOnce>(gs, dy + row * ldg);
        S.template load<kOnce>(ts, total + row * ldt);
        S.template load<kOnce>(as, dtotal + row * lda);
        S.template load<kOnce>(xs, x + row * P.ldx);
    };
    const uint64_t on = (uint64_t)gridDim.x * TEAMS;
    uint64_t first = (uint64_t)blockIdx.x * TEAMS;
    if constexpr (kAhead)
        load(first + team);
    Vectors V{kept};
    if (threadIdx.x < (uint32_t)TEAM) {
        float a[NV][VEC], b[NV][VEC];
        vector_or<W>(a, P.w2, S, 1.0f);
        V.put(0, a);
        vector_or<W>(a, P.gate, S, 1.0f);
        vector_or<W>(b, kInner ? P.w1 : nullptr, S, 1.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                a[k][e] = a[k][e] * P.factor * b[k][e];
        V.put(1, a);
    }
    __syncthreads();
    // (teams of several waves meet at barriers in every row: a workgroup's teams take equally many turns)
    for (; first < P.rows; first += on) {
        const uint64_t row = first + team;
        if (row >= P.rows) {                                 // (the workgroup's last turn: only barriers are left to meet)
            if constexpr (TEAM > 64) {
                __syncthreads();
                if constexpr (kInner)
                    __syncthreads();
            }
            break;
        }
        if constexpr (!kAhead)
            load(row);
        float d[NV][VEC], n[NV][VEC], w[NV][VEC];
        Vec<T, VEC> through_sum[NV], branch[NV];             // (of the row; the arrays above are the next one's from here on)
        const float m1 = P.inner == kLayerNorm ? mean1 : 0.0f, r1 = rstd1, m2 = P.outer == kLayerNorm ? mean2 : 0.0f, r2 = rstd2;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            through_sum[k] = as[k];
            branch[k] = xs[k];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                n[k][e] = ((float)ts[k][e] - m2) * r2;
                d[k][e] = (float)gs[k][e];
            }
        }
        if constexpr (TEAM > 64) {
            arrived(through_sum);
            // (without an inner norm x is in no sum before the one barrier behind which dx is stored: dx may be x, and where a row is not
            // whole vectors another wave's last vector has columns of this thread's)
            if constexpr (kSums && !kInner)
                arrived(branch);
        }
        if constexpr (kAhead)
            load(row + on);
        if (outer) {
            if constexpr (kSums)
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        total_of[2][k][e] = __builtin_fmaf(d[k][e], n[k][e], total_of[2][k][e]);
                        total_of[3][k][e] += d[k][e];
                    }
            V.get(0, w);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    d[k][e] *= w[k][e];
            Pair sum = add_up<Shape, NV, VEC>(S, whole, [&](int k, int e, Pair &p) {
                p.a += d[k][e];
                p.b = __builtin_fmaf(d[k][e], n[k][e], p.b);
            });
            row_sums<TEAM, WAVES>(sum.a, sum.b, red, turn);
            sum.a = P.outer == kLayerNorm ? sum.a * per : 0.0f;
            sum.b *= per;
            if constexpr (!kSums)
                if (P.means && threadIdx.x % TEAM == 0) {
                    P.means[row] = sum.a;
                    P.means[P.rows + row] = sum.b;
                }
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    d[k][e] = __builtin_fmaf(-n[k][e], sum.b, d[k][e] - sum.a);
                    d[k][e] = P.dtotal ? __builtin_fmaf(d[k][e], r2, (float)through_sum[k][e]) : d[k][e] * r2;
                }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    d[k][e] = (float)through_sum[k][e];
            if constexpr (TEAM > 64)
                __syncthreads();
        }
        if (P.dresidual) {                                   // (behind a barrier: dresidual may be dtotal or total)
            float through[NV][VEC];
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    through[k][e] = d[k][e] * P.residual_scale;
            S.template store<kOnce>(static_cast<T *>(P.dresidual) + row * P.lde, through);
        }
        if (P.draws.threshold) {                             // d is u from here on
            const BucketKey key = bucket_key(begin, row);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                drop<VEC>(d[k], key, S.at[k], P.draws.threshold);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                n[k][e] = kInner ? ((float)branch[k][e] - m1) * r1 : (float)branch[k][e];
                if constexpr (kSums) {
                    total_of[0][k][e] = __builtin_fmaf(d[k][e], n[k][e], total_of[0][k][e]);
                    if constexpr (kInner)
                        total_of[1][k][e] += d[k][e];
                }
            }
        V.get(1, w);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                d[k][e] *= w[k][e];
        if constexpr (kInner) {
            Pair sum = add_up<Shape, NV, VEC>(S, whole, [&](int k, int e, Pair &p) {
                p.a += d[k][e];
                p.b = __builtin_fmaf(d[k][e], n[k][e], p.b);
            });
            row_sums<TEAM, WAVES>(sum.a, sum.b, red, turn);
            sum.a = P.inner == kLayerNorm ? sum.a * per : 0.0f;
            sum.b *= per;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    d[k][e] = __builtin_fmaf(-n[k][e], sum.b, d[k][e] - sum.a) * r1;
        }
        S.template store<kOnce>(static_cast<T *>(P.dx) + row * P.ldd, d);
    }
    if constexpr (kSums) {
        float *const out = P.partial + (uint64_t)blockIdx.x * kSeamSums * hidden;
        if constexpr (TEAMS > 1) {                           // the workgroup's teams, in a fixed order
            constexpr int SETS = TEAM < 64 ? WAVES : TEAMS;  // (teams in one wave add up there)
            __shared__ float all[SETS][TEAM * E];
            const uint32_t set = threadIdx.x / (TEAM < 64 ? 64u : (uint32_t)TEAM);
#pragma unroll
            for (int which = 0; which < (int)kSeamSums; ++which) {
                __syncthreads();
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        float sum = total_of[which][k][e];
#pragma unroll
                        for (int off = TEAM; off < 64; off <<= 1)
                            sum += __shfl_xor(sum, off, 64);
                        if ((TEAM >= 64 || threadIdx.x % 64u < (uint32_t)TEAM) && S.counts(k, e))
                            all[set][S.at[k] + e] = sum;
                    }
                __syncthreads();
                for (uint32_t c = threadIdx.x; c < hidden; c += WG) {
                    float sum = all[0][c];
#pragma unroll
                    for (int k = 1; k < SETS; ++k)
                        sum += all[k][c];
                    out[which * hidden + c] = sum;
                }
            }
        } else {                                             // (a shared column: the same sum from both)
#pragma unroll
            for (int which = 0; which < (int)kSeamSums; ++which)
                S.store(out + which * hidden, total_of[which]);
        }
    }
}

// The same sums for rows whose team has no registers left for them: rows blockIdx.y, blockIdx.y + gridDim.y, ..., a vector of columns
// per thread, from the means that the launch before it left.  In pieces of 32 rows, which keep what rounding adds up to low.
template <class T, class W>
__global__ __launch_bounds__(256) void k_residual_norm_columns(const ResidualNormBackward P)
{
    constexpr int VEC = 16 / sizeof(T);
    const uint32_t col = (blockIdx.x * 256u + threadIdx.x) * VEC;
    if (col >= P.hidden)
        return;
    const uint32_t at = min(col, P.hidden - VEC);
    const bool outer = P.outer != kNoNorm, inner = P.inner != kNoNorm;
    const uint64_t begin = P.draws.begin();
    float w2[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        w2[e] = 1.0f;
    if (P.w2)
        load_as_float<VEC>(w2, static_cast<const W *>(P.w2) + at);
    float total_of[kSeamSums][VEC] = {};
    for (uint64_t row = blockIdx.y; row < P.rows;) {
        float part[kSeamSums][VEC] = {};
        for (uint32_t k = 0; k < 32u && row < P.rows; ++k, row += gridDim.y) {
            float d[VEC] = {}, n[VEC], a[VEC] = {};
            if (P.dtotal)
                load_as_float<VEC>(a, static_cast<const T *>(P.dtotal) + row * P.lda + at);
            if (outer) {
                const float mean = P.outer == kLayerNorm ? P.stats[2u * P.rows + row] : 0.0f, rstd = P.stats[3u * P.rows + row];
                const float s1 = P.means[row], s2 = P.means[P.rows + row];
                load_as_float<VEC>(d, static_cast<const T *>(P.dy) + row * P.ldg + at);
                load_as_float<VEC>(n, static_cast<const T *>(P.total) + row * P.ldt + at);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    n[e] = (n[e] - mean) * rstd;
                    part[2][e] = __builtin_fmaf(d[e], n[e], part[2][e]);
                    part[3][e] += d[e];
                    d[e] = __builtin_fmaf(-n[e], s2, d[e] * w2[e] - s1) * rstd;
                }
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                d[e] += a[e];
            if (P.draws.threshold)
                drop<VEC>(d, bucket_key(begin, row), at, P.draws.threshold);
            load_as_float<VEC>(n, static_cast<const T *>(P.x) + row * P.ldx + at);
            const float mean = P.inner == kLayerNorm ? P.stats[row] : 0.0f, rstd = inner ? P.stats[P.rows + row] : 1.0f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                part[0][e] = __builtin_fmaf(d[e], (n[e] - mean) * rstd, part[0][e]);
                part[1][e] += d[e];
            }
        }
#pragma unroll
        for (uint32_t which = 0; which < kSeamSums; ++which)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                total_of[which][e] += part[which][e];
    }
    float *const out = P.partial + (uint64_t)blockIdx.y * kSeamSums * P.hidden + at;
#pragma unroll
    for (uint32_t which = 0; which < kSeamSums; ++which)     // (a shared column: the same sum from both)
        store_from_float<VEC>(out + which * P.hidden, total_of[which]);
}

struct SeamVectors {
    const void *w1, *b1, *gate;                              // each may be none
    void *dw1, *db1, *dgate, *dw2, *db2;                     // each may be none
    float factor;
};

// The gradients of the vectors from the partial sums: blockIdx.y 0 those of the branch, 1 dw2 and db2.
template <class W>
__global__ __launch_bounds__(1024) void k_residual_norm_finish(const float *partial, uint32_t parts, uint32_t hidden, const SeamVectors V)
{
    const uint64_t stride = (uint64_t)kSeamSums * hidden;
    if (blockIdx.y == 1u) {
        if (V.dw2 || V.db2)
            column_totals<2>(partial + 2u * hidden, stride, parts, hidden, [&](uint32_t c, const float (&sum)[2]) {
                if (V.dw2)
                    static_cast<W *>(V.dw2)[c] = (W)sum[0];
                if (V.db2)
                    static_cast<W *>(V.db2)[c] = (W)sum[1];
            });
    } else if (V.dw1 || V.db1 || V.dgate) {
        column_totals<2>(partial, stride, parts, hidden, [&](uint32_t c, const float (&sum)[2]) {
            const auto of = [&](const void *v, float other) { return v ? (float)static_cast<const W *>(v)[c] : other; };
            const float g = of(V.gate, 1.0f) * V.factor;
            if (V.dw1)
                static_cast<W *>(V.dw1)[c] = (W)(g * sum[0]);
            if (V.db1)
                static_cast<W *>(V.db1)[c] = (W)(g * sum[1]);
            if (V.dgate)
                static_cast<W *>(V.dgate)[c] = (W)(V.factor * __builtin_fmaf(of(V.w1, 1.0f), sum[0], of(V.b1, 0.0f) * sum[1]));
        });
    }
}

}  // namespace nuq
