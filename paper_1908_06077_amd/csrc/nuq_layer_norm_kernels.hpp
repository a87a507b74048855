// Layer norm of rows, forward and backward.
//
//   s = x (+ residual), rounded to x's type;  mean, var over the row;  rstd = 1 / sqrt(var + eps)
//   n = (s - mean) rstd;  y = n weight + bias
//   d = dy weight;  dx = rstd (d - mean(d) - n mean(d n)) (+ add);  dweight = sum over rows of dy n;  dbias = sum of dy
//
// A row stays in the registers of one team of threads between its statistics and its result: read once, written once.  The
// variance is taken of the centred values.  Statistics and sums are fp32, results are rounded to their type once.
//
// Bound by HBM (counted: 1.00 to 1.01 times the bytes of the rows, and the partial sums), and on rows of a few KiB by latency:
// what a CU has in flight.  So teams are small (a wave has a row of 1024 elements, no barrier), at most sixteen elements per
// thread keep the registers low enough for several teams per CU, a team stays for many rows with the next one's loads issued
// before the present one's sums, and weight and bias are read once: read per row, 12.8 KB of them for each 3.2 KB row of 1600
// in bfloat16, they took the L1 7 us of a 26 us pass.  Plain accesses: with non-temporal stores the pass on 8192 x 1600 takes
// 18 us instead of 21.6, but an operation that reads both results behind it 19 instead of 13.
#pragma once

#include "nuq_train_device.hpp"

namespace nuq {

// How a team of TEAM threads holds a row: each has E elements, in vectors of VEC neighbouring ones (16 bytes, or single elements
// for rows shorter than that).  A thread whose vector would end behind the row takes the row's last VEC elements instead: its
// loads need no branch, it computes what a neighbour computes too for the elements they share, and leaves these out of sums.
template <class T, int TEAM_, int E, int VEC_>
struct RowShape {
    static constexpr int TEAM = TEAM_, VEC = VEC_, NV = E / VEC_;
    static_assert(E % VEC_ == 0, "whole vectors");
    uint32_t at[NV];            // first column of each vector
    uint32_t twice[NV];         // elements of it that a neighbour has too: VEC for a vector that is not there
    __device__ __forceinline__ explicit RowShape(uint32_t hidden)
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (uint32_t)(k * TEAM + (int)(threadIdx.x % TEAM)) * VEC;
            at[k] = min(col, hidden - VEC);
            twice[k] = min(col - at[k], (uint32_t)VEC);
        }
    }
    __device__ __forceinline__ bool there(int k) const { return twice[k] < (uint32_t)VEC; }
    __device__ __forceinline__ bool counts(int k, int e) const { return (uint32_t)e >= twice[k]; }
    // kOnce: with the hint that the memory is touched once.
    template <bool kOnce = false, class V>
    __device__ __forceinline__ void load(Vec<V, VEC> (&to)[NV], const V *row) const
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const auto *const from = reinterpret_cast<const Vec<V, VEC> *>(row + at[k]);
            if constexpr (kOnce)
                to[k] = __builtin_nontemporal_load(from);
            else
                to[k] = *from;
        }
    }
    template <bool kOnce = false, class V>
    __device__ __forceinline__ void store(V *row, const float (&from)[NV][VEC]) const
    {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (there(k))
                store_from_float<VEC, kOnce>(row + at[k], from[k]);
    }
};

struct LayerNormForward {
    const void *x, *residual, *weight, *bias;  // residual, weight, bias: may be none
    void *total, *y;                           // total: where there is a residual
    float *mean, *rstd;                        // may be none
    uint64_t rows, ldx, ldr, ldt, ldy;         // row strides in elements
    uint32_t hidden;
    float eps;
};

// Sum over the TEAM threads of a row, the same bits in each.  Teams of more than a wave: red holds a float per wave, and is
// not used again before another barrier.
template <int TEAM>
__device__ __forceinline__ float row_sum(float x, float *red)
{
    if constexpr (TEAM <= 64) {
        return team_sum<TEAM>(x);
    } else {
        x = team_sum<64>(x);
        if (threadIdx.x % 64u == 0)
            red[threadIdx.x / 64u] = x;
        __syncthreads();
        x = red[0];
#pragma unroll
        for (int k = 1; k < TEAM / 64; ++k)
            x += red[k];
        return x;
    }
}

// Threads of a workgroup: teams of more than a wave meet at barriers and have it alone.
template <int TEAM>
constexpr int kForwardWG = TEAM <= 64 ? 256 : TEAM;

// A team takes rows in turn; the next row is on its way while one is worked on, weight and bias stay in registers.  8192 x 1600 in
// bfloat16 with the residual 21.7 us (4.8 TB/s, of which 2 us are the launch), 8192 x 12288 in float32 142 us (5.7 TB/s), one row
// 2.1 us (a launch); one row per workgroup instead: 26.5 and 152 us.
template <class T, class W, int TEAM, int E, int VEC, bool kStream>
__global__ __launch_bounds__(kForwardWG<TEAM>) void k_layer_norm_forward(const LayerNormForward P)
{
    using Shape = RowShape<T, TEAM, E, VEC>;
    constexpr int NV = Shape::NV, TEAMS = kForwardWG<TEAM> / TEAM;
    __shared__ float red[2][TEAM > 64 ? TEAM / 64 : 1];
    const uint32_t hidden = P.hidden;
    const Shape S(hidden);
    const W *const weight = static_cast<const W *>(P.weight), *const bias = static_cast<const W *>(P.bias);
    uint64_t row = (uint64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM;
    if (row >= P.rows)                                       // (a whole team; teams of more than a wave are the workgroup)
        return;
    Vec<T, VEC> xs[NV], rs[NV];
    Vec<W, VEC> ws[NV], bs[NV];
    const auto load = [&]() {
        S.load(xs, static_cast<const T *>(P.x) + row * P.ldx);
        if constexpr (kStream)
            S.load(rs, static_cast<const T *>(P.residual) + row * P.ldr);
    };
    load();
    if (weight)
        S.load(ws, weight);
    if (bias)
        S.load(bs, bias);
    for (;;) {
        const uint64_t now = row;
        float s[NV][VEC], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                s[k][e] = (float)xs[k][e];
                if constexpr (kStream)
                    s[k][e] = (float)(T)(s[k][e] + (float)rs[k][e]);
                sum += S.counts(k, e) ? s[k][e] : 0.0f;
            }
        row += (uint64_t)gridDim.x * TEAMS;
        const bool more = row < P.rows;
        if (more)
            load();
        const float mean = row_sum<TEAM>(sum, red[0]) / (float)hidden;
        if constexpr (kStream)                               // (behind the barrier: total may be x or residual)
            S.store(static_cast<T *>(P.total) + now * P.ldt, s);
        float square = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                s[k][e] -= mean;
                square = __builtin_fmaf(S.counts(k, e) ? s[k][e] : 0.0f, s[k][e], square);
            }
        const float rstd = 1.0f / __builtin_sqrtf(row_sum<TEAM>(square, red[1]) / (float)hidden + P.eps);
        if (threadIdx.x % TEAM == 0) {
            if (P.mean)
                P.mean[now] = mean;
            if (P.rstd)
                P.rstd[now] = rstd;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                s[k][e] *= rstd;
                if (weight)
                    s[k][e] *= (float)ws[k][e];
                if (bias)
                    s[k][e] += (float)bs[k][e];
            }
        S.store(static_cast<T *>(P.y) + now * P.ldy, s);
        if (!more)
            break;
    }
}

// Rows that no team's registers hold: a workgroup reads its row three times, from cache where it fits (1024 x 32768 in bfloat16
// 44.5 us, 3.0 TB/s of the bytes of one reading, 107 us with single elements instead of 16 bytes).  A thread's part of a row has no
// bound, so it adds up in fp64 what its vectors sum to in fp32: the error does not grow with the row.
constexpr int kLongRowWG = 1024;

// f(first column, elements to leave out) for the thread's vectors of VEC neighbouring elements of a row of at least VEC.  The last
// vector of a row that is no multiple begins earlier; what it shares with its neighbour is left out.
template <int VEC, int WG, class F>
__device__ __forceinline__ void for_row(uint32_t hidden, F &&f)
{
    for (uint32_t col = threadIdx.x * VEC; col < hidden; col += WG * VEC) {
        const uint32_t at = min(col, hidden - VEC);
        f(at, col - at);
    }
}
template <int VEC, class T>
__device__ __forceinline__ void store_behind(T *to, const float (&from)[VEC], uint32_t skip)
{
    if (skip == 0) {
        store_from_float<VEC>(to, from);
    } else {
#pragma unroll
        for (int e = 1; e < VEC; ++e)
            if ((uint32_t)e >= skip)
                to[e] = (T)from[e];
    }
}

template <class T, class W, bool kStream>
__global__ __launch_bounds__(kLongRowWG) void k_layer_norm_forward_long(const LayerNormForward P)
{
    constexpr int VEC = 16 / sizeof(T);
    __shared__ float red[2][kLongRowWG / 64];
    for (uint64_t row = blockIdx.x; row < P.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(P.x) + row * P.ldx;
        double all = 0.0;
        if constexpr (kStream) {
            const T *const res = static_cast<const T *>(P.residual) + row * P.ldr;
            T *const total = static_cast<T *>(P.total) + row * P.ldt;
            for_row<VEC, kLongRowWG>(P.hidden, [&](uint32_t at, uint32_t skip) {
                float s[VEC], r[VEC];
                load_as_float<VEC>(s, x + at);
                load_as_float<VEC>(r, res + at);
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    s[e] = (float)(T)(s[e] + r[e]);
                    sum += (uint32_t)e >= skip ? s[e] : 0.0f;
                }
                all += sum;
                store_behind<VEC>(total + at, s, skip);          // (read again by the thread that wrote it)
            });
            x = total;
        } else {
            for_row<VEC, kLongRowWG>(P.hidden, [&](uint32_t at, uint32_t skip) {
                float s[VEC], sum = 0.0f;
                load_as_float<VEC>(s, x + at);
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    sum += (uint32_t)e >= skip ? s[e] : 0.0f;
                all += sum;
            });
        }
        const float mean = row_sum<kLongRowWG>((float)all, red[0]) / (float)P.hidden;
        all = 0.0;
        for_row<VEC, kLongRowWG>(P.hidden, [&](uint32_t at, uint32_t skip) {
            float s[VEC], square = 0.0f;
            load_as_float<VEC>(s, x + at);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float d = (uint32_t)e >= skip ? s[e] - mean : 0.0f;
                square = __builtin_fmaf(d, d, square);
            }
            all += square;
        });
        const float rstd = 1.0f / __builtin_sqrtf(row_sum<kLongRowWG>((float)all, red[1]) / (float)P.hidden + P.eps);
        if (threadIdx.x == 0) {
            if (P.mean)
                P.mean[row] = mean;
            if (P.rstd)
                P.rstd[row] = rstd;
        }
        T *const y = static_cast<T *>(P.y) + row * P.ldy;
        for_row<VEC, kLongRowWG>(P.hidden, [&](uint32_t at, uint32_t skip) {
            float n[VEC], w[VEC], b[VEC];
            load_as_float<VEC>(n, x + at);
            if (P.weight)
                load_as_float<VEC>(w, static_cast<const W *>(P.weight) + at);
            if (P.bias)
                load_as_float<VEC>(b, static_cast<const W *>(P.bias) + at);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                n[e] = (n[e] - mean) * rstd;
                if (P.weight)
                    n[e] *= w[e];
                if (P.bias)
                    n[e] += b[e];
            }
            store_behind<VEC>(y + at, n, skip);
        });
    }
}

struct LayerNormBackward {
    const void *dy, *x, *weight, *add;         // weight, add: may be none
    const float *mean, *rstd;
    void *dx;
    float *partial;                            // [parts][2][hidden] sums of dy n and of dy, or none
    uint64_t rows, ldg, ldx, lda, ldd;
    uint32_t hidden;
};

// Threads of a workgroup: more than one team shares what is written of the sums.  Eight elements per thread leave registers for
// sixteen waves (8192 x 1600 in bfloat16 25.7 us, 26.6 with two workgroups of eight), sixteen for eight (twelve were 4 % slower).
template <int TEAM, int E>
constexpr int kBackwardWG = TEAM < 512 ? (E <= 8 ? 1024 : 512) : TEAM;

// A team takes rows in turn, as in the forward pass, and keeps the sums of its columns in registers.  Workgroup p writes
// partial[p], 8 bytes per column; a second launch (4 to 12 us) adds the workgroups up.  8192 x 1600 in bfloat16 with a gradient to
// add 22.5 us (4.8 TB/s with the partial sums), 32768 x 8192 282 us (5.8 TB/s), 33554 x 1000 in float32 101 us (5.3), 4096 x 16384 in
// bfloat16, where one workgroup fills a CU, 84 us (4.8).  With sixteen elements per thread the sums and operands take 160 registers,
// so that a CU has eight waves; held to 128 they spill, and the pass takes twice as long; in LDS the sums cost 10 % (but win above
// 8192 columns).
template <class T, class W, int TEAM, int E, int VEC, bool kSums>
__global__ __launch_bounds__((kBackwardWG<TEAM, E>)) void k_layer_norm_backward(const LayerNormBackward P)
{
    using Shape = RowShape<T, TEAM, E, VEC>;
    constexpr int NV = Shape::NV, WG = kBackwardWG<TEAM, E>, TEAMS = WG / TEAM, WAVES = WG / 64, TEAM_WAVES = TEAM < 64 ? 1 : TEAM / 64;
    constexpr bool kAhead = TEAM < 1024;                     // (sixteen waves leave too few registers for a row ahead,
    constexpr bool kInLds = kSums && TEAM >= 768;            //  and twelve for the sums too: these stand in LDS then)
    __shared__ __align__(16) float kept[kInLds ? 2 * TEAM * E : 1];
    __shared__ float red[2][2][WAVES];
    const uint32_t hidden = P.hidden;
    const Shape S(hidden);
    const W *const weight = static_cast<const W *>(P.weight);
    const float per = 1.0f / (float)hidden;
    float dw[NV][VEC] = {}, db[NV][VEC] = {};
    // a thread's own places in LDS
    const auto kept_at = [&](int which, int k) { return kept + ((which * NV + k) * TEAM + (int)(threadIdx.x % TEAM)) * VEC; };
    if constexpr (kInLds)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            store_from_float<VEC>(kept_at(0, k), dw[k]);
            store_from_float<VEC>(kept_at(1, k), db[k]);
        }
    uint32_t turn = 0;
    Vec<T, VEC> xs[NV], gs[NV], as[NV];
    Vec<W, VEC> ws[NV];
    float mean = 0.0f, rstd = 0.0f;
    uint64_t row = (uint64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM;
    const auto load = [&]() {
        mean = P.mean[row];
        rstd = P.rstd[row];
        S.load(gs, static_cast<const T *>(P.dy) + row * P.ldg);
        S.load(xs, static_cast<const T *>(P.x) + row * P.ldx);
    };
    const auto load_add = [&](uint64_t of) {                 // (used last in a row, so asked for when the last one is used)
        if (P.add)
            S.load(as, static_cast<const T *>(P.add) + of * P.lda);
    };
    if (kAhead && row < P.rows) {
        load();
        load_add(row);
    }
    if (weight)
        S.load(ws, weight);
    // (teams of several waves meet at a barrier in every row: a workgroup's teams take equally many turns)
    for (uint64_t first = (uint64_t)blockIdx.x * TEAMS; first < P.rows; first += (uint64_t)gridDim.x * TEAMS) {
        const uint64_t now = row;
        if (TEAM <= 64 && now >= P.rows)
            break;
        if (!kAhead && now < P.rows)
            load();
        if (TEAM > 64 && now >= P.rows) {                    // (only the barrier is left to meet)
            __syncthreads();
            break;
        }
        const float scale = rstd;
        float n[NV][VEC], d[NV][VEC], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if constexpr (kInLds) {
                load_as_float<VEC>(dw[k], kept_at(0, k));
                load_as_float<VEC>(db[k], kept_at(1, k));
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                n[k][e] = ((float)xs[k][e] - mean) * rstd;
                d[k][e] = (float)gs[k][e];
                if constexpr (kSums) {
                    dw[k][e] = __builtin_fmaf(d[k][e], n[k][e], dw[k][e]);
                    db[k][e] += d[k][e];
                }
                if (weight)
                    d[k][e] *= (float)ws[k][e];
                const float c = S.counts(k, e) ? d[k][e] : 0.0f;
                s1 += c;
                s2 = __builtin_fmaf(c, n[k][e], s2);
            }
            if constexpr (kInLds) {
                store_from_float<VEC>(kept_at(0, k), dw[k]);
                store_from_float<VEC>(kept_at(1, k), db[k]);
            }
        }
        row += (uint64_t)gridDim.x * TEAMS;
        if (kAhead && row < P.rows)
            load();
        if (!kAhead)
            load_add(now);
        if constexpr (TEAM <= 64) {
            s1 = team_sum<TEAM>(s1);
            s2 = team_sum<TEAM>(s2);
        } else {
            s1 = team_sum<64>(s1);
            s2 = team_sum<64>(s2);
            if (threadIdx.x % 64u == 0) {
                red[turn][0][threadIdx.x / 64u] = s1;
                red[turn][1][threadIdx.x / 64u] = s2;
            }
            __syncthreads();                                 // (two sets of sums: one barrier per row)
            const uint32_t own = threadIdx.x / TEAM * TEAM_WAVES;
            s1 = red[turn][0][own];
            s2 = red[turn][1][own];
#pragma unroll
            for (int k = 1; k < TEAM_WAVES; ++k) {
                s1 += red[turn][0][own + k];
                s2 += red[turn][1][own + k];
            }
            turn ^= 1u;
        }
        s1 *= per;
        s2 *= per;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                d[k][e] = (d[k][e] - s1 - n[k][e] * s2) * scale;
                if (P.add)
                    d[k][e] += (float)as[k][e];
            }
        if (kAhead && row < P.rows)
            load_add(row);
        S.store(static_cast<T *>(P.dx) + now * P.ldd, d);
    }
    if constexpr (kSums) {
        if constexpr (kInLds)
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                load_as_float<VEC>(dw[k], kept_at(0, k));
                load_as_float<VEC>(db[k], kept_at(1, k));
            }
        float *const out = P.partial + (uint64_t)blockIdx.x * 2u * hidden;
        if constexpr (TEAMS > 1) {                           // the workgroup's teams, in a fixed order
            constexpr int SETS = TEAM < 64 ? WAVES : TEAMS;  // (teams in one wave add up there)
            __shared__ float all[SETS][TEAM * E];
            const uint32_t set = threadIdx.x / (TEAM < 64 ? 64u : (uint32_t)TEAM);
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                if (which)
                    __syncthreads();
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        float sum = which ? db[k][e] : dw[k][e];
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
            S.store(out, dw);
            S.store(out + hidden, db);
        }
    }
}

template <class T, class W>
__global__ __launch_bounds__(kLongRowWG) void k_layer_norm_backward_long(const LayerNormBackward P)
{
    constexpr int VEC = 16 / sizeof(T);
    __shared__ float red[2][kLongRowWG / 64];
    for (uint64_t row = blockIdx.x; row < P.rows; row += gridDim.x) {
        const T *const x = static_cast<const T *>(P.x) + row * P.ldx;
        const T *const dy = static_cast<const T *>(P.dy) + row * P.ldg;
        const float mean = P.mean[row], rstd = P.rstd[row];
        const auto both = [&](uint32_t at, float (&n)[VEC], float (&d)[VEC]) {
            float w[VEC];
            load_as_float<VEC>(n, x + at);
            load_as_float<VEC>(d, dy + at);
            if (P.weight)
                load_as_float<VEC>(w, static_cast<const W *>(P.weight) + at);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                n[e] = (n[e] - mean) * rstd;
                if (P.weight)
                    d[e] *= w[e];
            }
        };
        double all1 = 0.0, all2 = 0.0;
        for_row<VEC, kLongRowWG>(P.hidden, [&](uint32_t at, uint32_t skip) {
            float n[VEC], d[VEC], s1 = 0.0f, s2 = 0.0f;
            both(at, n, d);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float c = (uint32_t)e >= skip ? d[e] : 0.0f;
                s1 += c;
                s2 = __builtin_fmaf(c, n[e], s2);
            }
            all1 += s1;
            all2 += s2;
        });
        const float s1 = row_sum<kLongRowWG>((float)all1, red[0]) / (float)P.hidden;
        const float s2 = row_sum<kLongRowWG>((float)all2, red[1]) / (float)P.hidden;
        T *const dx = static_cast<T *>(P.dx) + row * P.ldd;
        for_row<VEC, kLongRowWG>(P.hidden, [&](uint32_t at, uint32_t skip) {
            float n[VEC], d[VEC], a[VEC];
            both(at, n, d);
            if (P.add)
                load_as_float<VEC>(a, static_cast<const T *>(P.add) + row * P.lda + at);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                d[e] = (d[e] - s1 - n[e] * s2) * rstd;
                if (P.add)
                    d[e] += a[e];
            }
            store_behind<VEC>(dx + at, d, skip);
        });
    }
}

// Sums over rows blockIdx.y, blockIdx.y + gridDim.y, ... of the long rows, a vector of columns per thread; in pieces of 32 rows, which
// keep what rounding adds up to at 32 and a 2048th of the rows.
template <class T>
__global__ __launch_bounds__(256) void k_layer_norm_columns(const LayerNormBackward P)
{
    constexpr int VEC = 16 / sizeof(T);
    const uint32_t col = (blockIdx.x * 256u + threadIdx.x) * VEC;
    if (col >= P.hidden)
        return;
    const uint32_t at = min(col, P.hidden - VEC);
    float dw[VEC] = {}, db[VEC] = {};
    for (uint64_t row = blockIdx.y; row < P.rows;) {
        float w[VEC] = {}, b[VEC] = {};
        for (uint32_t k = 0; k < 32u && row < P.rows; ++k, row += gridDim.y) {
            float n[VEC], d[VEC];
            load_as_float<VEC>(d, static_cast<const T *>(P.dy) + row * P.ldg + at);
            load_as_float<VEC>(n, static_cast<const T *>(P.x) + row * P.ldx + at);
            const float mean = P.mean[row], rstd = P.rstd[row];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                w[e] = __builtin_fmaf(d[e], (n[e] - mean) * rstd, w[e]);
                b[e] += d[e];
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            dw[e] += w[e];
            db[e] += b[e];
        }
    }
    float *const out = P.partial + (uint64_t)blockIdx.y * 2u * P.hidden + at;
    store_from_float<VEC>(out, dw);                          // (a shared column: the same sum from both)
    store_from_float<VEC>(out + P.hidden, db);
}

// put(column, sums) for the sums of `parts` vectors of `hidden` floats that stand `stride` floats apart, of K such sets that stand one
// behind the other, in a fixed order: 16 columns at a time per workgroup of 1024, 64 threads to each.
template <int K, class F>
__device__ __forceinline__ void column_totals(const float *partial, uint64_t stride, uint32_t parts, uint32_t hidden, F &&put)
{
    __shared__ float red[K][64][17];
    const uint32_t c = threadIdx.x % 16u, group = threadIdx.x / 16u;
    for (uint32_t begin = blockIdx.x * 16u;;) {
        const uint32_t col = begin + c;
        float sum[K] = {};
        if (col < hidden) {
            const float *const from = partial + col;
            uint32_t p = group;
            for (; p + 192u < parts; p += 256u) {            // four loads of each at once
                float x[K][4];
#pragma unroll
                for (int i = 0; i < K; ++i)
#pragma unroll
                    for (uint32_t k = 0; k < 4u; ++k)
                        x[i][k] = from[(p + 64u * k) * stride + (uint32_t)i * hidden];
#pragma unroll
                for (int i = 0; i < K; ++i)
                    sum[i] += (x[i][0] + x[i][1]) + (x[i][2] + x[i][3]);
            }
            for (; p < parts; p += 64u)
#pragma unroll
                for (int i = 0; i < K; ++i)
                    sum[i] += from[p * stride + (uint32_t)i * hidden];
        }
#pragma unroll
        for (int i = 0; i < K; ++i)
            red[i][group][c] = sum[i];
        __syncthreads();
        if (threadIdx.x < 64u) {                             // one wave: four lanes to a column
            const uint32_t cc = threadIdx.x / 4u, part = threadIdx.x % 4u, to = begin + cc;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                sum[i] = 0.0f;
#pragma unroll
                for (uint32_t k = 0; k < 16u; ++k)
                    sum[i] += red[i][part * 16u + k][cc];
                sum[i] = team_sum<4>(sum[i]);
            }
            if (part == 0 && to < hidden)
                put(to, sum);
        }
        begin += gridDim.x * 16u;                            // (hidden is at most 2^30, a grid's columns 2^24)
        if (begin >= hidden)
            break;
        __syncthreads();
    }
}

// dweight and dbias (blockIdx.y) from the partial sums.
template <class W>
__global__ __launch_bounds__(1024) void k_layer_norm_finish(const float *partial, uint32_t parts, uint32_t hidden, W *dweight,
                                                            W *dbias)
{
    W *const out = blockIdx.y ? dbias : dweight;
    if (out)
        column_totals<1>(partial + (uint64_t)blockIdx.y * hidden, 2ull * hidden, parts, hidden,
                         [&](uint32_t c, const float (&sum)[1]) { out[c] = (W)sum[0]; });
}

}  // namespace nuq
