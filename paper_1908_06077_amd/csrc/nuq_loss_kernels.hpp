// Softmax cross entropy of rows x against the weights w of a large vocabulary, with its gradients; the logits z = x w^T are never in
// memory.
//
//   lse = log sum over v of exp(z_v);  loss = lse - (1 - e) z_t - e mean(z)          (t the target, e the smoothing)
//   d_v = exp(z_v - lse) - e / V - (1 - e) [v = t];  dx = g d w;  dw = sum over rows of g d x        (g the loss's gradient)
//
// Forward a workgroup makes a tile of logits on the matrix cores and leaves two numbers per row and group of the vocabulary, the
// largest logit and the sum of exp(z - largest); a second launch joins them.  Backward the vocabulary goes through in pieces: a
// launch makes a piece's logits again and writes d, rounded to the operands' type (its products sum over rows or the vocabulary in
// fp32, and a rounding of up to 2^-8 or 2^-11 of each term is what the operands have too); two products take it to dx and dw.  Exponentials
// are exp2 of a product with log2 e: a term e^-t of a sum is off by t e^-t 2^-24 more, 0.4 2^-24 of the largest at most.
// Bound by the matrix cores: 2 N V H operations forward, 6 N V H backward and 2 N V H for the logits made again; on few rows by reading w.
// Measured in bfloat16, H = 1600, V = 50257: 8192 rows forward 970 to 1023 us (1.29 to 1.36 PFLOP/s; 1045 is what a library product of
// the same shape takes that does write the logits), backward 3360 to 3487 us (1.51 to 1.57 PFLOP/s over its four products); one row forward
// 34 us, w at 5.0 TB/s.  The results of a tile (nine vector instructions and an exponential per logit) hide nothing: all waves of a CU are at
// them at once.  Fewer were tried, without the comparisons where a block has no target and no end: forward 1013 -> 1024, so these stay.
#pragma once

#include "nuq_product_device.hpp"
#include "nuq_train_device.hpp"

namespace nuq {

constexpr float kLog2E = 1.44269504088896340736f;

// What d is multiplied with before it is rounded: of a vocabulary of 50000 most d are near 2^-16, where fp16 has two bits left.
template <class T>
constexpr float kGradientScale = __is_same(T, _Float16) ? 0x1p14f : 1.0f;

// Rows of the caller or of the workspace: stride in bytes, a multiple of 16.
struct LossOperands {
    const void *x, *w;
    uint32_t stride_x, stride_w, chunks;       // chunks: 16-byte pieces of a row
    uint32_t rows, vocab;
    uint32_t mt, nt;                           // tiles
};

struct LossForward {
    LossOperands O;
    const int64_t *target;
    float2 *part;                              // [tiles of the vocabulary][rows]: largest logit, sum of exp(z - largest)
    float *sums;                               // the same: sum of logits, where targets are smoothed
    float *of_target;                          // [rows]: the target's logit
};

// The tiles of logits that a workgroup makes: every gridDim.x-th, the first step of the next one on its way while one is worked on.
template <class Tile>
struct LogitTiles {
    const LossOperands &O;
    uint32_t id, m0, n0;
    __device__ __forceinline__ LogitTiles(const LossOperands &o, Tile &tile) : O(o), id(blockIdx.x) { begin(tile); }
    __device__ __forceinline__ void begin(Tile &tile)
    {
        tile_of(id, O.mt, O.nt, m0, n0);
        m0 *= Tile::BM;
        n0 *= Tile::BN;
        tile.begin({static_cast<const char *>(O.w) + (uint64_t)m0 * O.stride_w, O.stride_w, min((uint32_t)Tile::BM, O.vocab - m0), O.chunks},
                   {static_cast<const char *>(O.x) + (uint64_t)n0 * O.stride_x, O.stride_x, min((uint32_t)Tile::BN, O.rows - n0), O.chunks},
                   (O.chunks + 7u) / 8u);
    }
    // Whether there is another tile, which is begun.
    __device__ __forceinline__ bool next(Tile &tile)
    {
        id += gridDim.x;
        const bool more = id < O.mt * O.nt;
        if (more)
            begin(tile);
        return more;
    }
};

// The sum of exp(z - base) needs a base that is finite.
__device__ __forceinline__ float finite_base(float top) { return __builtin_isinf(top) ? 0.0f : top; }

// Largest logit, sum of exp(z - largest) and sum of logits of a part of the vocabulary.
struct LossPart {
    float top, sum, all;
    __device__ __forceinline__ void join(float other, float its, float logits)
    {
        const float higher = fmaxf(top, other), base = finite_base(higher);
        sum = sum * __builtin_amdgcn_exp2f((top - base) * kLog2E) + its * __builtin_amdgcn_exp2f((other - base) * kLog2E);
        top = higher;
        all += logits;
    }
    // Over the wave's first WIDTH lanes, the same in each.
    template <int WIDTH>
    __device__ __forceinline__ void join_lanes()
    {
#pragma unroll
        for (int off = 1; off < WIDTH; off <<= 1)
            join(__shfl_xor(top, off, 64), __shfl_xor(sum, off, 64), __shfl_xor(all, off, 64));
    }
};

template <class T, class Tile, bool kSmooth>
__global__ __launch_bounds__(Tile::THREADS) void k_loss_logits(const LossForward P)
{
    __shared__ __align__(16) char lds[Tile::LDS];
    constexpr uint32_t WIDE = Tile::BM / Tile::WM;           // of a wave
    static_assert(Tile::BN <= Tile::THREADS && sizeof(LossPart) * Tile::BN * Tile::WM <= Tile::STAGE, "a row's parts");
    Tile tile(lds);
    LogitTiles<Tile> tiles(P.O, tile);
    for (bool more = true; more;) {
        const uint32_t m0 = tiles.m0, n0 = tiles.n0, mw = m0 + tile.first_m();
        tile.run();
        const uint32_t thread = thread_again(), quad = thread / 16u % 4u * 4u, nw = n0 + tile.first_n() + thread % 16u;
        uint32_t target[Tile::NI];                           // (the lane's columns of a block are quad to quad + 3)
#pragma unroll
        for (int j = 0; j < Tile::NI; ++j) {
            const int64_t t = nw + j * 16u < P.O.rows ? P.target[nw + j * 16u] : -1;
            target[j] = (uint64_t)t < P.O.vocab ? (uint32_t)t : ~0u;
        }
        more = tiles.next(tile);
        tile.finish();
        // (what the lane's columns are compared with is moved by the lane's place, not the columns: those would fill the registers)
        const uint32_t there = mw < P.O.vocab ? min(WIDE, P.O.vocab - mw) : 0u;
        const int32_t lane_there = (int32_t)(there - quad);
        LossPart part[Tile::NI];
#pragma unroll
        for (int j = 0; j < Tile::NI; ++j) {
            const uint32_t at = target[j] - mw < there ? target[j] - mw : ~0u, lane_at = at - quad;
            float top = -__builtin_inff(), sum = 0.0f, all = 0.0f, wanted = 0.0f;
#pragma unroll
            for (int i = 0; i < Tile::MI; ++i) {
                if (i % 4 == 0)
                    __builtin_amdgcn_sched_barrier(0);       // (four blocks after the other: there are no registers for more)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t m = i * 16u + r;
                    float z = tile.acc[i][j][r];
                    if (m == lane_at)
                        wanted = z;
                    if constexpr (kSmooth)
                        all += (int32_t)m < lane_there ? z : 0.0f;
                    z = (int32_t)m < lane_there ? z : -__builtin_inff();
                    tile.acc[i][j][r] = z;
                    top = fmaxf(top, z);
                }
            }
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float base = finite_base(top);
#pragma unroll
            for (int i = 0; i < Tile::MI; ++i) {
                if (i % 4 == 0)
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    sum += __builtin_amdgcn_exp2f((tile.acc[i][j][r] - base) * kLog2E);
            }
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if constexpr (kSmooth) {
                all += __shfl_xor(all, 16, 64);
                all += __shfl_xor(all, 32, 64);
            }
            if (at != ~0u && (at & 12u) == quad)
                P.of_target[nw + j * 16u] = wanted;
            part[j] = {top, sum, all};
        }
        // the waves that have parts of one row, joined by a thread of the row
        LossPart *const parts = reinterpret_cast<LossPart *>(tile.free_stage());
#pragma unroll
        for (int j = 0; j < Tile::NI; ++j)
            if (quad == 0u)
                parts[(mw - m0) / WIDE * Tile::BN + tile.first_n() + j * 16u + thread % 16u] = part[j];
        lds_barrier();
        const uint32_t n = n0 + thread;
        if (thread < (uint32_t)Tile::BN && n < P.O.rows) {
            LossPart p = parts[thread];
#pragma unroll
            for (int k = 1; k < Tile::WM; ++k) {
                const LossPart q = parts[k * Tile::BN + thread];
                p.join(q.top, q.sum, q.all);
            }
            const uint64_t to = (uint64_t)(m0 / Tile::BM) * P.O.rows + n;
            P.part[to] = make_float2(p.top, p.sum);
            if constexpr (kSmooth)
                P.sums[to] = p.all;
        }
    }
}

struct LossJoin {
    const int64_t *target;
    const float2 *part;
    const float *sums, *of_target;             // sums: where targets are smoothed
    float *row_loss, *lse;
    float *mean;                               // [2], may be none: the mean loss, and 1 / rows that count
    uint32_t *flags;
    int64_t ignore;
    uint32_t rows, vocab, groups;
    float smoothing;
};

// The mean over the rows that count, in a fixed order in fp64, by one workgroup of 1024.
__device__ __forceinline__ void loss_mean(const LossJoin &P)
{
    __shared__ double red[2][16];
    double sum = 0.0, count = 0.0;
#pragma unroll 4
    for (uint32_t n = threadIdx.x; n < P.rows; n += 1024u) {
        const int64_t target = P.target[n];
        const float loss = P.row_loss[n];
        sum += target != P.ignore ? (double)loss : 0.0;
        count += target != P.ignore ? 1.0 : 0.0;
    }
    sum = workgroup_sum<1024>(sum, red[0]);
    count = workgroup_sum<1024>(count, red[1]);
    if (threadIdx.x == 0) {
        const double part = count > 0.0 ? 1.0 / count : 1.0;
        P.mean[0] = (float)(sum * part);
        P.mean[1] = (float)part;
    }
}

// ROWS rows per workgroup (1 or 16), 1024 / ROWS threads to each.  kAlone: there are no more rows, and the mean is taken here.
template <int ROWS, bool kAlone>
__global__ __launch_bounds__(1024) void k_loss_join(const LossJoin P)
{
    constexpr uint32_t THREADS = 1024 / ROWS;
    static_assert(ROWS == 1 || ROWS == 16, "a wave per row, or sixteen");
    __shared__ LossPart parts[ROWS][ROWS == 1 ? 16 : 65];
    const uint32_t r = threadIdx.x % ROWS, of = threadIdx.x / ROWS, lane = threadIdx.x % 64u, wave = threadIdx.x / 64u;
    uint32_t n = blockIdx.x * ROWS + r;
    LossPart p{-__builtin_inff(), 0.0f, 0.0f};
    if (n < P.rows)
#pragma unroll 4
        for (uint32_t g = of; g < P.groups; g += THREADS) {
            const float2 x = P.part[(uint64_t)g * P.rows + n];
            p.join(x.x, x.y, P.sums ? P.sums[(uint64_t)g * P.rows + n] : 0.0f);
        }
    bool writes;                                             // the one thread that has all of row n
    if constexpr (ROWS == 1) {
        p.join_lanes<64>();
        if (lane == 0)
            parts[0][wave] = p;
        __syncthreads();
        p = parts[0][lane % 16u];
        p.join_lanes<16>();
        writes = threadIdx.x == 0;
    } else {                                                 // wave k joins what row k's 64 threads have
        parts[r][of] = p;
        __syncthreads();
        p = parts[wave][lane];
        p.join_lanes<64>();
        n = blockIdx.x * ROWS + wave;
        writes = lane == 0;
    }
    if (writes && n < P.rows) {
        const float lse = p.top == __builtin_inff() && p.sum == p.sum ? p.top : finite_base(p.top) + logf(p.sum);
        const int64_t t = P.target[n];
        float loss = 0.0f;
        if (t != P.ignore) {
            if (t >= 0 && t < (int64_t)P.vocab) {
                loss = (1.0f - P.smoothing) * (lse - P.of_target[n]);
                if (P.sums)
                    loss += P.smoothing * (lse - p.all / (float)P.vocab);
            } else {
                loss = __builtin_nanf("");
                atomicOr(P.flags, (uint32_t)NUQ_FLAG_MALFORMED);
            }
        }
        P.lse[n] = lse;
        P.row_loss[n] = loss;
    }
    if constexpr (kAlone) {
        if (!P.mean)
            return;
        __syncthreads();                                     // (one workgroup: it reads what it wrote)
        loss_mean(P);
    }
}

__global__ __launch_bounds__(1024) void k_loss_mean(const LossJoin P) { loss_mean(P); }

// Per row what the gradients need: the target, or -1 for a row without one; g over the largest |g|; g over the gradients' scale.
struct LossRows {
    const int64_t *target;
    const float *grad, *mean;                  // grad: one number, or one per row; mean: may be none, mean[1] is multiplied in
    int32_t *code;
    float *factor, *scale;
    float *largest;                            // [1]: the largest |g| of a row that counts, over the gradients' scale
    uint32_t *flags;
    int64_t ignore;
    uint32_t rows, vocab;
    bool per_row;
    float inverse;                             // of the gradients' scale
    // (A row that does not count has gradient 0, whatever the caller's is: a NaN of its loss may have come back.)
    __device__ __forceinline__ bool counts(int64_t t) const { return t != ignore && t >= 0 && t < (int64_t)vocab; }
};

// One workgroup where there is a gradient per row, whose largest is sought; as many as there are thousands of rows elsewhere.
__global__ __launch_bounds__(1024) void k_loss_rows(const LossRows P)
{
    __shared__ float tops[16];
    const float part = P.mean ? P.mean[1] : 1.0f;
    float top = 0.0f;
    if (P.per_row) {
        bool lost = false;
        for (uint32_t n = threadIdx.x; n < P.rows; n += 1024u)
            if (P.counts(P.target[n])) {
                const float g = fabsf(P.grad[n] * part);
                lost |= !(g < __builtin_inff());
                top = fmaxf(top, g);
            }
        top = lost ? __builtin_nanf("") : top;
        for (int off = 32; off > 0; off >>= 1) {
            const float other = __shfl_xor(top, off, 64);
            top = top == top && !(other <= top) ? other : top;
        }
        if (threadIdx.x % 64u == 0)
            tops[threadIdx.x / 64u] = top;
        __syncthreads();
        for (int k = 0; k < 16; ++k)
            top = top == top && !(tops[k] <= top) ? tops[k] : top;
    } else {
        top = P.grad[0] * part;
    }
    bool bad = false;
    for (uint32_t n = blockIdx.x * 1024u + threadIdx.x; n < P.rows; n += gridDim.x * 1024u) {
        int32_t code = -1;
        float factor = 0.0f, scale = 0.0f;
        const int64_t t = P.target[n];
        if (P.counts(t)) {
            code = (int32_t)t;
            const float g = P.per_row ? P.grad[n] * part : top;
            factor = !P.per_row ? 1.0f : top == 0.0f ? 0.0f : g / top;
            scale = g * P.inverse;
        } else if (t != P.ignore) {
            bad = true;
        }
        P.code[n] = code;
        P.factor[n] = factor;
        P.scale[n] = scale;
    }
    if (bad)
        atomicOr(P.flags, (uint32_t)NUQ_FLAG_MALFORMED);
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *P.largest = top * P.inverse;
}

// Rows as the products take them: at a stride that is a multiple of 16 bytes, zeros behind their end.  With a code, zeros for a row without
// a target, whatever it holds, and the others times their factor.
template <class T>
__global__ __launch_bounds__(256) void k_loss_pack(const T *from, uint64_t ld, uint64_t rows, uint32_t columns, T *to, uint32_t to_ld,
                                                   const int32_t *code, const float *factor)
{
    constexpr uint32_t VEC = 16u / sizeof(T);
    const uint32_t per = to_ld / VEC;
    for (uint64_t v = (uint64_t)blockIdx.x * 256u + threadIdx.x; v < rows * per; v += (uint64_t)gridDim.x * 256u) {
        const uint64_t row = v / per;
        const uint32_t at = (uint32_t)(v % per) * VEC;
        float x[VEC] = {};
        if (!code || code[row] >= 0) {
            load_some<(int)VEC>(x, from + row * ld + at, (int64_t)columns - at);
            if (code)
#pragma unroll
                for (uint32_t e = 0; e < VEC; ++e)
                    x[e] *= factor[row];
        }
        store_from_float<(int)VEC>(to + row * to_ld + at, x);
    }
}

struct LossGradient {
    LossOperands O;                            // w, vocab: of the piece
    const int32_t *code;
    const float *lse;
    void *d;                                   // [rows][piece padded to 64], zeros behind the piece
    uint32_t first;                            // of the vocabulary
    uint32_t padded_vocab;
    float smoothed, wanted;                    // e / V, 1 - e
};

template <class T, class Tile>
__global__ __launch_bounds__(Tile::THREADS) void k_loss_gradient(const LossGradient P)
{
    __shared__ __align__(16) char lds[Tile::LDS];
    Tile tile(lds);
    LogitTiles<Tile> tiles(P.O, tile);
    for (bool more = true; more;) {
        const uint32_t mw = tiles.m0 + tile.first_m(), n0 = tiles.n0 + tile.first_n();
        tile.run();
        const uint32_t thread = thread_again(), quad = thread / 16u % 4u * 4u;
        int32_t code[Tile::NI];
        float lse[Tile::NI];
#pragma unroll
        for (int j = 0; j < Tile::NI; ++j) {
            const uint32_t n = n0 + j * 16u + thread % 16u;
            code[j] = n < P.O.rows ? P.code[n] : -1;
            lse[j] = n < P.O.rows ? P.lse[n] : 0.0f;
        }
        more = tiles.next(tile);
        tile.finish();
        // d of columns quad to quad + 3 of block i, of the lane's row of block j
        const auto gradient = [&](int j, int i, float (&x)[4]) {
            const uint32_t m = i * 16u, target = (uint32_t)code[j] - P.first - mw - quad;            // (none in the piece: no place in it)
            const int32_t there = code[j] >= 0 ? (int32_t)(P.O.vocab - mw - quad) : 0;
#pragma unroll
            for (uint32_t e = 0; e < 4u; ++e) {
                float v = __builtin_amdgcn_exp2f((tile.acc[i][j][e] - lse[j]) * kLog2E) - P.smoothed;
                if (m + e == target)
                    v -= P.wanted;
                x[e] = (int32_t)(m + e) < there ? v * kGradientScale<T> : 0.0f;
            }
        };
        const auto row = [&](int j, uint32_t r) -> T * {
            const uint32_t n = n0 + j * 16u + r;
            return n < P.O.rows ? static_cast<T *>(P.d) + (uint64_t)n * P.padded_vocab + mw : nullptr;
        };
        if constexpr (sizeof(T) == 2) {
            tile.store_rows(gradient, row, (int64_t)P.padded_vocab - mw);
        } else {
#pragma unroll
            for (int j = 0; j < Tile::NI; ++j)
#pragma unroll
                for (int i = 0; i < Tile::MI; ++i) {
                    float x[4];
                    gradient(j, i, x);
                    T *const to = row(j, threadIdx.x % 16u);
                    if (to && mw + i * 16u < P.padded_vocab)
                        store_from_float<4>(to + i * 16 + quad, x);
                }
        }
    }
}

// out[n][m] (+)= sum over k of a[k][m] b[n][k] (or b[k][n], where Tile takes that operand across) times *scale, for m below `columns` and n
// below `rows`; workgroups of split s take `each` of the k from s * each on and write the s-th of the outputs.
struct LossProduct {
    const void *a, *b;
    uint32_t stride_a, stride_b;               // bytes
    uint32_t wide_a, wide_b;                   // across: 16-byte pieces of a row
    uint32_t deep_a, deep_b, each;             // k that there are in either, at least one split's
    uint32_t columns, rows, mt, nt;
    void *out;
    uint64_t ld, next;                         // elements from row to row, from split to split
    const float *scale;
};

template <class T, class Tile, class O, bool kAcrossB, bool kAdd>
__global__ __launch_bounds__(Tile::THREADS) void k_loss_product(const LossProduct P)
{
    __shared__ __align__(16) char lds[Tile::LDS];
    constexpr uint32_t VEC = 16u / (uint32_t)sizeof(T);
    const uint32_t all = P.mt * P.nt, split = blockIdx.x / all, quad = threadIdx.x / 16u % 4u * 4u;
    uint32_t bm, bn;
    tile_of(blockIdx.x % all, P.mt, P.nt, bm, bn);
    const uint32_t m0 = bm * Tile::BM, n0 = bn * Tile::BN, k0 = split * P.each;
    const auto left = [&](uint32_t deep) -> uint32_t { return k0 < deep ? min(P.each, deep - k0) : 0u; };
    const auto across = [&](const void *p, uint32_t stride, uint32_t wide, uint32_t deep, uint32_t first, uint32_t size) -> Operand {
        const uint32_t pieces = min(size / VEC, wide - first / VEC);
        return {static_cast<const char *>(p) + (uint64_t)k0 * stride + (uint64_t)first * sizeof(T), stride, pieces, left(deep)};
    };
    const float scale = P.scale ? *P.scale : 1.0f;
    Tile tile(lds);
    constexpr uint32_t DEPTH = 128u / (uint32_t)sizeof(T);
    const Operand a = across(P.a, P.stride_a, P.wide_a, P.deep_a, m0, Tile::BM);
    const uint32_t steps = max(1u, (left(max(P.deep_a, P.deep_b)) + DEPTH - 1u) / DEPTH);
    if constexpr (kAcrossB)
        tile.begin(a, across(P.b, P.stride_b, P.wide_b, P.deep_b, n0, Tile::BN), steps);
    else
        tile.begin(a, {static_cast<const char *>(P.b) + (uint64_t)n0 * P.stride_b + (uint64_t)k0 * sizeof(T), P.stride_b,
                       min((uint32_t)Tile::BN, P.rows - n0), left(P.deep_b) / VEC}, steps);
    tile.run();
    tile.finish();
    const uint32_t mw = m0 + tile.first_m();
    O *const out = static_cast<O *>(P.out) + split * P.next + mw;
    const auto row = [&](int j, uint32_t r) -> O * {
        const uint32_t n = n0 + tile.first_n() + j * 16u + r;
        return n < P.rows ? out + n * P.ld : nullptr;
    };
    if constexpr (sizeof(O) == 2 && !kAdd) {
        tile.store_rows([&](int j, int i, float (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = tile.acc[i][j][e] * scale;
        }, row, (int64_t)P.columns - mw);
    } else {
#pragma unroll
        for (int j = 0; j < Tile::NI; ++j) {
            O *const to = row(j, threadIdx.x % 16u);
            if (!to)
                continue;
#pragma unroll
            for (int i = 0; i < Tile::MI; ++i) {
                const uint32_t m = i * 16u + quad;
                const int64_t have = (int64_t)P.columns - mw - m;
                if (have <= 0)
                    continue;
                float x[4], before[4] = {};
                if constexpr (kAdd)
                    load_some<4>(before, to + m, have);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] = tile.acc[i][j][e] * scale + before[e];
                store_some<4>(to + m, x, have);
            }
        }
    }
}

// dx[n][m] <- scale[n] times the sum of the splits; 0 in a row without a target.
template <class T>
__global__ __launch_bounds__(256) void k_loss_rows_gradient(const float *sums, uint64_t ld, uint64_t next, uint32_t splits,
                                                            const int32_t *code, const float *scale, uint32_t rows, uint32_t hidden,
                                                            T *dx, uint64_t ldd)
{
    const uint32_t per = (hidden + 3u) / 4u;
    for (uint64_t v = (uint64_t)blockIdx.x * 256u + threadIdx.x; v < (uint64_t)rows * per; v += (uint64_t)gridDim.x * 256u) {
        const uint32_t n = (uint32_t)(v / per), at = (uint32_t)(v % per) * 4u;
        float x[4] = {};
        if (code[n] >= 0) {
            for (uint32_t s = 0; s < splits; ++s) {
                float y[4];
                load_as_float<4>(y, sums + s * next + n * ld + at);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] += y[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] *= scale[n];
        }
        store_some<4>(dx + n * ldd + at, x, (int64_t)hidden - at);
    }
}

}  // namespace nuq
