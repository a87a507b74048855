// Layer norm of rows, forward and backward.
//
//   s = x (+ residual), rounded to x's type;  mean, var over the row;  rstd = 1 / sqrt(var + eps)
//   n = (s - mean) rstd;  y = n weight + bias
//   d = dy weight;  dx = rstd (d - mean(d) - n mean(d n)) (+ add);  dweight = sum over rows of dy n;  dbias = sum of dy
//
// A row stays in the registers of one team of threads between its statistics and its result: read once, written once.  The
// variance is taken of the centred values.  Statistics and sums are fp32, results are rounded to their type once.
#pragma once

#include "nuq_train_device.hpp"

namespace nuq {

template <class T>
constexpr int kVecOf = 16 / sizeof(T);         // elements of a 16-byte access

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

template <class T, class W, int TEAM, int NV, bool kStream>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void k_layer_norm_forward(const LayerNormForward P)
{
    constexpr int VEC = kVecOf<T>, WG = TEAM < 256 ? 256 : TEAM;
    __shared__ float red[2][TEAM > 64 ? TEAM / 64 : 1];
    const uint64_t row = (uint64_t)blockIdx.x * (WG / TEAM) + threadIdx.x / TEAM;
    if (row >= P.rows)                                       // (a whole team; teams of more than a wave are the workgroup)
        return;
    const uint32_t lane = threadIdx.x % TEAM;
    const T *const x = static_cast<const T *>(P.x) + row * P.ldx;
    float s[NV][VEC], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t col = (k * TEAM + lane) * VEC;
        load_some<VEC>(s[k], x + col, (int64_t)P.hidden - col);
    }
    if constexpr (kStream) {
        const T *const res = static_cast<const T *>(P.residual) + row * P.ldr;
        T *const total = static_cast<T *>(P.total) + row * P.ldt;
        float r[NV][VEC];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (k * TEAM + lane) * VEC;
            load_some<VEC>(r[k], res + col, (int64_t)P.hidden - col);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (k * TEAM + lane) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s[k][e] = (float)(T)(s[k][e] + r[k][e]);
            store_some<VEC>(total + col, s[k], (int64_t)P.hidden - col);
        }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            sum += s[k][e];
    const float mean = row_sum<TEAM>(sum, red[0]) / (float)P.hidden;
    float square = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t col = (k * TEAM + lane) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            s[k][e] = col + e < P.hidden ? s[k][e] - mean : 0.0f;
            square = __builtin_fmaf(s[k][e], s[k][e], square);
        }
    }
    const float rstd = 1.0f / __builtin_sqrtf(row_sum<TEAM>(square, red[1]) / (float)P.hidden + P.eps);
    if (lane == 0) {
        if (P.mean)
            P.mean[row] = mean;
        if (P.rstd)
            P.rstd[row] = rstd;
    }
    T *const y = static_cast<T *>(P.y) + row * P.ldy;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t col = (k * TEAM + lane) * VEC;
        const int64_t have = (int64_t)P.hidden - col;
        float w[VEC], b[VEC];
        if (P.weight)
            load_some<VEC>(w, static_cast<const W *>(P.weight) + col, have);
        if (P.bias)
            load_some<VEC>(b, static_cast<const W *>(P.bias) + col, have);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            s[k][e] *= rstd;
            if (P.weight)
                s[k][e] *= w[e];
            if (P.bias)
                s[k][e] += b[e];
        }
        store_some<VEC>(y + col, s[k], have);
    }
}

// Rows that no team's registers hold: a workgroup reads its row three times (from cache, where it fits).
constexpr int kLongRowWG = 1024;

template <class T, class W, bool kStream>
__global__ __launch_bounds__(kLongRowWG) void k_layer_norm_forward_long(const LayerNormForward P)
{
    __shared__ float red[2][kLongRowWG / 64];
    const uint64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(P.x) + row * P.ldx;
    float sum = 0.0f;
    if constexpr (kStream) {
        const T *const res = static_cast<const T *>(P.residual) + row * P.ldr;
        T *const total = static_cast<T *>(P.total) + row * P.ldt;
        for (uint32_t col = threadIdx.x; col < P.hidden; col += kLongRowWG) {
            const T t = (T)((float)x[col] + (float)res[col]);
            total[col] = t;                                  // (read again by the thread that wrote it)
            sum += (float)t;
        }
        x = total;
    } else {
        for (uint32_t col = threadIdx.x; col < P.hidden; col += kLongRowWG)
            sum += (float)x[col];
    }
    const float mean = row_sum<kLongRowWG>(sum, red[0]) / (float)P.hidden;
    float square = 0.0f;
    for (uint32_t col = threadIdx.x; col < P.hidden; col += kLongRowWG) {
        const float d = (float)x[col] - mean;
        square = __builtin_fmaf(d, d, square);
    }
    const float rstd = 1.0f / __builtin_sqrtf(row_sum<kLongRowWG>(square, red[1]) / (float)P.hidden + P.eps);
    if (threadIdx.x == 0) {
        if (P.mean)
            P.mean[row] = mean;
        if (P.rstd)
            P.rstd[row] = rstd;
    }
    T *const y = static_cast<T *>(P.y) + row * P.ldy;
    for (uint32_t col = threadIdx.x; col < P.hidden; col += kLongRowWG) {
        float n = ((float)x[col] - mean) * rstd;
        if (P.weight)
            n *= (float)static_cast<const W *>(P.weight)[col];
        if (P.bias)
            n += (float)static_cast<const W *>(P.bias)[col];
        y[col] = (T)n;
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

// Workgroup p takes rows p, p + parts, ... of each of its teams' strides and writes partial[p].
template <class T, class W, int TEAM, int NV, bool kSums>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void k_layer_norm_backward(const LayerNormBackward P)
{
    constexpr int VEC = kVecOf<T>, WG = TEAM < 256 ? 256 : TEAM, TEAMS = WG / TEAM, WAVES = WG / 64;
    __shared__ float red[2][2][WAVES];
    const uint32_t lane = threadIdx.x % TEAM;
    float dw[NV][VEC] = {}, db[NV][VEC] = {};
    uint32_t turn = 0;
    for (uint64_t row = (uint64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM; row < P.rows; row += (uint64_t)gridDim.x * TEAMS) {
        const T *const x = static_cast<const T *>(P.x) + row * P.ldx;
        const T *const dy = static_cast<const T *>(P.dy) + row * P.ldg;
        const float mean = P.mean[row], rstd = P.rstd[row];
        float n[NV][VEC], d[NV][VEC], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (k * TEAM + lane) * VEC;
            load_some<VEC>(n[k], x + col, (int64_t)P.hidden - col);
            load_some<VEC>(d[k], dy + col, (int64_t)P.hidden - col);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (k * TEAM + lane) * VEC;
            float w[VEC];
            if (P.weight)
                load_some<VEC>(w, static_cast<const W *>(P.weight) + col, (int64_t)P.hidden - col);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                n[k][e] = (n[k][e] - mean) * rstd;           // (beyond the row dy is 0, and so is what is made of it)
                if constexpr (kSums) {
                    dw[k][e] = __builtin_fmaf(d[k][e], n[k][e], dw[k][e]);
                    db[k][e] += d[k][e];
                }
                if (P.weight)
                    d[k][e] *= w[e];
                s1 += d[k][e];
                s2 = __builtin_fmaf(d[k][e], n[k][e], s2);
            }
        }
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
            s1 = red[turn][0][0];
            s2 = red[turn][1][0];
#pragma unroll
            for (int k = 1; k < WAVES; ++k) {
                s1 += red[turn][0][k];
                s2 += red[turn][1][k];
            }
            turn ^= 1u;
        }
        s1 /= (float)P.hidden;
        s2 /= (float)P.hidden;
        T *const dx = static_cast<T *>(P.dx) + row * P.ldd;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (k * TEAM + lane) * VEC;
            const int64_t have = (int64_t)P.hidden - col;
            float a[VEC];
            if (P.add)
                load_some<VEC>(a, static_cast<const T *>(P.add) + row * P.lda + col, have);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                d[k][e] = (d[k][e] - s1 - n[k][e] * s2) * rstd;
                if (P.add)
                    d[k][e] += a[e];
            }
            store_some<VEC>(dx + col, d[k], have);
        }
    }
    if constexpr (kSums) {
        float *const out = P.partial + (uint64_t)blockIdx.x * 2u * P.hidden;
        if constexpr (TEAM <= 64) {                          // the workgroup's teams, in a fixed order
            constexpr int COLS = NV * TEAM * VEC;
            __shared__ float all[WAVES][2][COLS];
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
#pragma unroll
                    for (int off = TEAM; off < 64; off <<= 1) {
                        dw[k][e] += __shfl_xor(dw[k][e], off, 64);
                        db[k][e] += __shfl_xor(db[k][e], off, 64);
                    }
                    if (threadIdx.x % 64u < TEAM) {
                        all[threadIdx.x / 64u][0][(k * TEAM + lane) * VEC + e] = dw[k][e];
                        all[threadIdx.x / 64u][1][(k * TEAM + lane) * VEC + e] = db[k][e];
                    }
                }
            __syncthreads();
            for (uint32_t c = threadIdx.x; c < P.hidden; c += WG)
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    float sum = all[0][which][c];
#pragma unroll
                    for (int k = 1; k < WAVES; ++k)
                        sum += all[k][which][c];
                    out[which * P.hidden + c] = sum;
                }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const uint32_t col = (k * TEAM + lane) * VEC;
                store_some<VEC>(out + col, dw[k], (int64_t)P.hidden - col);
                store_some<VEC>(out + P.hidden + col, db[k], (int64_t)P.hidden - col);
            }
        }
    }
}

template <class T, class W>
__global__ __launch_bounds__(kLongRowWG) void k_layer_norm_backward_long(const LayerNormBackward P)
{
    __shared__ float red[2][kLongRowWG / 64];
    const uint64_t row = blockIdx.x;
    const T *const x = static_cast<const T *>(P.x) + row * P.ldx;
    const T *const dy = static_cast<const T *>(P.dy) + row * P.ldg;
    const float mean = P.mean[row], rstd = P.rstd[row];
    auto both = [&](uint32_t col, float &n, float &d) {
        n = ((float)x[col] - mean) * rstd;
        d = (float)dy[col];
        if (P.weight)
            d *= (float)static_cast<const W *>(P.weight)[col];
    };
    float s1 = 0.0f, s2 = 0.0f, n, d;
    for (uint32_t col = threadIdx.x; col < P.hidden; col += kLongRowWG) {
        both(col, n, d);
        s1 += d;
        s2 = __builtin_fmaf(d, n, s2);
    }
    s1 = row_sum<kLongRowWG>(s1, red[0]) / (float)P.hidden;
    s2 = row_sum<kLongRowWG>(s2, red[1]) / (float)P.hidden;
    T *const dx = static_cast<T *>(P.dx) + row * P.ldd;
    for (uint32_t col = threadIdx.x; col < P.hidden; col += kLongRowWG) {
        both(col, n, d);
        d = (d - s1 - n * s2) * rstd;
        if (P.add)
            d += (float)static_cast<const T *>(P.add)[row * P.lda + col];
        dx[col] = (T)d;
    }
}

// Sums over rows blockIdx.y, blockIdx.y + gridDim.y, ... of the long rows, a column per thread.
template <class T>
__global__ __launch_bounds__(256) void k_layer_norm_columns(const LayerNormBackward P)
{
    const uint32_t col = blockIdx.x * 256u + threadIdx.x;
    if (col >= P.hidden)
        return;
    float dw = 0.0f, db = 0.0f;
    for (uint64_t row = blockIdx.y; row < P.rows; row += gridDim.y) {
        const float d = (float)static_cast<const T *>(P.dy)[row * P.ldg + col];
        const float n = ((float)static_cast<const T *>(P.x)[row * P.ldx + col] - P.mean[row]) * P.rstd[row];
        dw = __builtin_fmaf(d, n, dw);
        db += d;
    }
    P.partial[(uint64_t)blockIdx.y * 2u * P.hidden + col] = dw;
    P.partial[(uint64_t)blockIdx.y * 2u * P.hidden + P.hidden + col] = db;
}

// dweight and dbias (blockIdx.y) from the partial sums, in a fixed order: 64 columns per workgroup, 16 threads to each.
template <class W>
__global__ __launch_bounds__(1024) void k_layer_norm_finish(const float *partial, uint32_t parts, uint32_t hidden, W *dweight,
                                                            W *dbias)
{
    __shared__ float red[16][64];
    W *const out = blockIdx.y ? dbias : dweight;
    if (!out)
        return;
    const uint32_t col = blockIdx.x * 64u + threadIdx.x % 64u, group = threadIdx.x / 64u;
    float sum = 0.0f;
    if (col < hidden)
        for (uint32_t p = group; p < parts; p += 16u)
            sum += partial[((uint64_t)p * 2u + blockIdx.y) * hidden + col];
    red[group][threadIdx.x % 64u] = sum;
    __syncthreads();
    if (group == 0 && col < hidden) {
#pragma unroll
        for (int k = 1; k < 16; ++k)
            sum += red[k][threadIdx.x % 64u];
        out[col] = (W)sum;
    }
}

}  // namespace nuq
