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
// A row stays in the registers of one team of threads from its loads to its results: two rows are read and two written forward,
// four read and two written backward, whatever is fused.  Statistics and sums are fp32, the variance is taken of centred values,
// results are rounded to their type once.  The mask is computed again in the backward pass.  Bound by HBM, and on short batches by
// latency.
#pragma once

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
    float eps, scale, residual_scale;
};

// Sums over the threads of a row, one after the other: a set of red is not written again before a barrier that follows its last read,
// because the two sets take turns.
template <int TEAM>
struct RowSums {
    float (&red)[2][TEAM > 64 ? TEAM / 64 : 1];
    uint32_t turn;
    __device__ __forceinline__ float operator()(float x)
    {
        turn ^= 1u;
        return row_sum<TEAM>(x, red[turn]);
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

// A vector of `hidden` weights, which may be none, beside a team's row: in registers for all rows, or read again where it is used.
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
    __device__ __forceinline__ void multiply(const Shape &S, float (&s)[NV][VEC]) const
    {
        apply(S, [&](int k, int e, float w) { s[k][e] *= w; });
    }
    __device__ __forceinline__ void add(const Shape &S, float (&s)[NV][VEC]) const
    {
        apply(S, [&](int k, int e, float w) { s[k][e] += w; });
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

// Threads of a workgroup.
template <int TEAM>
constexpr int kSeamForwardWG = TEAM <= 64 ? 256 : TEAM;

// s <- N(s), its mean and reciprocal deviation.  between(): behind the first barrier, before s changes.
template <int TEAM, class Shape, int NV, int VEC, class F>
__device__ __forceinline__ void norm_row(float (&s)[NV][VEC], const Shape &S, RowSums<TEAM> &sums, uint32_t kind, float per, float eps,
                                         float &mean, float &rstd, F &&between)
{
    mean = 0.0f;
    if (kind == kLayerNorm) {
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                sum += S.counts(k, e) ? s[k][e] : 0.0f;
        mean = sums(sum) * per;
        between();
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s[k][e] -= mean;
    }
    float square = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            square = __builtin_fmaf(S.counts(k, e) ? s[k][e] : 0.0f, s[k][e], square);
    rstd = 1.0f / __builtin_sqrtf(sums(square) * per + eps);
    if (kind != kLayerNorm)
        between();
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            s[k][e] *= rstd;
}

template <class T, class W, int TEAM, int E, int VEC, bool kInner>
__global__ __launch_bounds__(kSeamForwardWG<TEAM>) void k_residual_norm_forward(const ResidualNormForward P)
{
    using Shape = RowShape<T, TEAM, E, VEC>;
    constexpr int NV = Shape::NV, TEAMS = kSeamForwardWG<TEAM> / TEAM;
    // the vectors of weights, and the next row ahead, in registers: not beside sixteen elements
    constexpr bool kHold = E <= 8, kAhead = E <= 8;
    __shared__ float red[2][TEAM > 64 ? TEAM / 64 : 1];
    const uint32_t hidden = P.hidden;
    const float per = 1.0f / (float)hidden;
    const Shape S(hidden);
    RowSums<TEAM> sums{red, 0u};
    uint32_t team = threadIdx.x / TEAM;
    if constexpr (TEAM >= 64)
        team = uniform_u32(team);
    uint64_t row = (uint64_t)blockIdx.x * TEAMS + team;
    if (row >= P.rows)                                       // (a whole team; teams of more than a wave are the workgroup)
        return;
    const uint64_t begin = P.draws.begin();
    Vec<T, VEC> xs[NV], rs[NV];
    const auto load = [&]() {
        S.load(xs, static_cast<const T *>(P.x) + row * P.ldx);
        S.load(rs, static_cast<const T *>(P.residual ? P.residual : P.x) + row * (P.residual ? P.ldr : P.ldx));
    };
    if constexpr (kAhead)
        load();
    using Weights = RowVector<Shape, W, NV, VEC, kHold>;
    const Weights w1(kInner ? P.w1 : nullptr, S), b1(kInner ? P.b1 : nullptr, S), gate(P.gate, S), w2(P.w2, S), b2(P.b2, S);
    for (;;) {
        const uint64_t now = row;
        if constexpr (!kAhead)
            load();
        float s[NV][VEC], mean, rstd;
        Vec<T, VEC> r[NV];
        if constexpr (TEAM > 64)
            arrived(rs);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            r[k] = rs[k];
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s[k][e] = (float)xs[k][e];
        }
        row += (uint64_t)gridDim.x * TEAMS;
        const bool more = row < P.rows;
        if (kAhead && more)
            load();
        if constexpr (kInner) {
            norm_row<TEAM>(s, S, sums, P.inner, per, P.eps, mean, rstd, [] {});
            if (P.stats && threadIdx.x % TEAM == 0) {
                if (P.inner == kLayerNorm)
                    P.stats[now] = mean;
                P.stats[P.rows + now] = rstd;
            }
            w1.multiply(S, s);
            b1.add(S, s);
        }
        gate.multiply(S, s);
        if (P.draws.threshold) {
            const BucketKey key = bucket_key(begin, now);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                drop<VEC>(s[k], key, S.at[k], P.draws.threshold, P.draws.keep);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s[k][e] = (float)(T)(s[k][e] * P.scale + (P.residual ? (float)r[k][e] * P.residual_scale : 0.0f));
        if (P.outer == kNoNorm) {                            // (behind a barrier of the inner norm: total may be x or residual)
            S.store(static_cast<T *>(P.total) + now * P.ldt, s);
        } else {
            norm_row<TEAM>(s, S, sums, P.outer, per, P.eps, mean, rstd, [&] { S.store(static_cast<T *>(P.total) + now * P.ldt, s); });
            if (P.stats && threadIdx.x % TEAM == 0) {
                if (P.outer == kLayerNorm)
                    P.stats[2u * P.rows + now] = mean;
                P.stats[3u * P.rows + now] = rstd;
            }
            w2.multiply(S, s);
            b2.add(S, s);
            S.store(static_cast<T *>(P.y) + now * P.ldy, s);
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
    float *partial;                            // [parts][5][hidden]: sums of h n, of h, of g n', of dy n2, of dy; or none
    float *means;                              // [2][rows] or none: mean(d), mean(d n2), for the sums that a launch of its own takes
    Draws draws;
    uint64_t rows, ldg, lda, ldx, ldt, ldd, lde;
    uint32_t hidden, inner, outer;
    float scale, residual_scale;
};
constexpr uint32_t kSeamSums = 5;

template <int TEAM>
constexpr int kSeamBackwardWG = TEAM <= 64 ? 256 : TEAM <= 512 ? 512 : TEAM;

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

// kSums: with the sums over rows, in registers; workgroup p writes partial[p], and a second launch adds those up.
template <class T, class W, int TEAM, int E, int VEC, bool kInner, bool kSums>
__global__ __launch_bounds__(kSeamBackwardWG<TEAM>) void k_residual_norm_backward(const ResidualNormBackward P)
{
    using Shape = RowShape<T, TEAM, E, VEC>;
    constexpr int NV = Shape::NV, WG = kSeamBackwardWG<TEAM>, TEAMS = WG / TEAM, WAVES = WG / 64;
    constexpr bool kHold = E <= 8;                           // (the vectors of weights, and all operands at once: not beside sixteen elements)
    __shared__ float red[2][2][WAVES];
    const uint32_t hidden = P.hidden;
    const Shape S(hidden);
    const float per = 1.0f / (float)hidden;
    const bool outer = P.outer != kNoNorm;
    uint32_t turn = 0, team = threadIdx.x / TEAM;
    if constexpr (TEAM >= 64)
        team = uniform_u32(team);
    const uint64_t begin = P.draws.begin();
    float total_of[kSeamSums][NV][VEC] = {};
    using Weights = RowVector<Shape, W, NV, VEC, kHold>;
    const Weights w1(kInner ? P.w1 : nullptr, S), b1(kInner && kSums ? P.b1 : nullptr, S), gate(P.gate, S), w2(P.w2, S);
    // (teams of several waves meet at barriers in every row: a workgroup's teams take equally many turns)
    for (uint64_t first = (uint64_t)blockIdx.x * TEAMS; first < P.rows; first += (uint64_t)gridDim.x * TEAMS) {
        const uint64_t row = first + team;
        if (row >= P.rows) {                                 // (the workgroup's last turn: only barriers are left to meet)
            if constexpr (TEAM > 64) {
                __syncthreads();
                if constexpr (kInner)
                    __syncthreads();
            }
            break;
        }
        Vec<T, VEC> xs[NV], as[NV];
        const auto load_x = [&]() { S.load(xs, static_cast<const T *>(P.x) + row * P.ldx); };
        float d[NV][VEC], n[NV][VEC];
        if (outer) {
            Vec<T, VEC> gs[NV], ts[NV];
            S.load(gs, static_cast<const T *>(P.dy) + row * P.ldg);
            S.load(ts, static_cast<const T *>(P.total) + row * P.ldt);
            // (without a gradient through the sum, dy in its place: read, and not added)
            S.load(as, static_cast<const T *>(P.dtotal ? P.dtotal : P.dy) + row * (P.dtotal ? P.lda : P.ldg));
            if constexpr (kHold && (kInner || kSums))
                load_x();
            const float mean = P.outer == kLayerNorm ? P.stats[2u * P.rows + row] : 0.0f, rstd = P.stats[3u * P.rows + row];
            float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    n[k][e] = ((float)ts[k][e] - mean) * rstd;
                    d[k][e] = (float)gs[k][e];
                    if constexpr (kSums) {
                        total_of[3][k][e] = __builtin_fmaf(d[k][e], n[k][e], total_of[3][k][e]);
                        total_of[4][k][e] += d[k][e];
                    }
                }
            w2.multiply(S, d);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float c = S.counts(k, e) ? d[k][e] : 0.0f;
                    s1 += c;
                    s2 = __builtin_fmaf(c, n[k][e], s2);
                }
            if constexpr (TEAM > 64)
                arrived(as);
            row_sums<TEAM, WAVES>(s1, s2, red, turn);
            s1 = P.outer == kLayerNorm ? s1 * per : 0.0f;
            s2 *= per;
            if (P.means && threadIdx.x % TEAM == 0) {
                P.means[row] = s1;
                P.means[P.rows + row] = s2;
            }
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    d[k][e] = (d[k][e] - s1 - n[k][e] * s2) * rstd + (P.dtotal ? (float)as[k][e] : 0.0f);
        } else {
            S.load(as, static_cast<const T *>(P.dtotal) + row * P.lda);
            if constexpr (kHold && (kInner || kSums))
                load_x();
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    d[k][e] = (float)as[k][e];
            if constexpr (TEAM > 64) {
                arrived(as);
                __syncthreads();
            }
        }
        if (P.dresidual) {                                   // (behind a barrier: dresidual may be dtotal or total)
            float through[NV][VEC];
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    through[k][e] = d[k][e] * P.residual_scale;
            S.store(static_cast<T *>(P.dresidual) + row * P.lde, through);
        }
        if constexpr (!kHold && (kInner || kSums))
            load_x();
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                d[k][e] *= P.scale;
        if (P.draws.threshold) {
            const BucketKey key = bucket_key(begin, row);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                drop<VEC>(d[k], key, S.at[k], P.draws.threshold, P.draws.keep);
        }
        if constexpr (kInner) {
            const float mean = P.inner == kLayerNorm ? P.stats[row] : 0.0f, rstd = P.stats[P.rows + row];
            float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    n[k][e] = ((float)xs[k][e] - mean) * rstd;
            if constexpr (kSums) {
                float whole[NV][VEC];
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        whole[k][e] = n[k][e];
                w1.multiply(S, whole);
                b1.add(S, whole);
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        total_of[2][k][e] = __builtin_fmaf(d[k][e], whole[k][e], total_of[2][k][e]);
            }
            gate.multiply(S, d);
            if constexpr (kSums)
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        total_of[0][k][e] = __builtin_fmaf(d[k][e], n[k][e], total_of[0][k][e]);
                        total_of[1][k][e] += d[k][e];
                    }
            w1.multiply(S, d);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float c = S.counts(k, e) ? d[k][e] : 0.0f;
                    s1 += c;
                    s2 = __builtin_fmaf(c, n[k][e], s2);
                }
            row_sums<TEAM, WAVES>(s1, s2, red, turn);
            s1 = P.inner == kLayerNorm ? s1 * per : 0.0f;
            s2 *= per;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    d[k][e] = (d[k][e] - s1 - n[k][e] * s2) * rstd;
        } else {
            if constexpr (kSums)
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        total_of[2][k][e] = __builtin_fmaf(d[k][e], (float)xs[k][e], total_of[2][k][e]);
            gate.multiply(S, d);
        }
        S.store(static_cast<T *>(P.dx) + row * P.ldd, d);
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
    float w1[VEC], b1[VEC] = {}, gate[VEC], w2[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        w1[e] = gate[e] = w2[e] = 1.0f;
    if (P.w1)
        load_as_float<VEC>(w1, static_cast<const W *>(P.w1) + at);
    if (P.b1)
        load_as_float<VEC>(b1, static_cast<const W *>(P.b1) + at);
    if (P.gate)
        load_as_float<VEC>(gate, static_cast<const W *>(P.gate) + at);
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
                    part[3][e] = __builtin_fmaf(d[e], n[e], part[3][e]);
                    part[4][e] += d[e];
                    d[e] = (d[e] * w2[e] - s1 - n[e] * s2) * rstd;
                }
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                d[e] = (d[e] + a[e]) * P.scale;
            if (P.draws.threshold)
                drop<VEC>(d, bucket_key(begin, row), at, P.draws.threshold, P.draws.keep);
            load_as_float<VEC>(n, static_cast<const T *>(P.x) + row * P.ldx + at);
            const float mean = P.inner == kLayerNorm ? P.stats[row] : 0.0f, rstd = inner ? P.stats[P.rows + row] : 1.0f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                n[e] = (n[e] - mean) * rstd;
                part[2][e] = __builtin_fmaf(d[e], n[e] * w1[e] + b1[e], part[2][e]);
                d[e] *= gate[e];
                part[0][e] = __builtin_fmaf(d[e], n[e], part[0][e]);
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
    void *to[kSeamSums];                                     // dw1, db1, dgate, dw2, db2; each may be none
};

template <class W>
__global__ __launch_bounds__(1024) void k_residual_norm_finish(const float *partial, uint32_t parts, uint32_t hidden, const SeamVectors V)
{
    column_totals(partial + (uint64_t)blockIdx.y * hidden, (uint64_t)kSeamSums * hidden, parts, hidden,
                  static_cast<W *>(V.to[blockIdx.y]));
}

}  // namespace nuq
