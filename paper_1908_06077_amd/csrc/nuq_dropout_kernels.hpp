// Dropout from the counter hash of the quantizer: the mask of element (r, c) of rows is a function of seed, step, r and c, computed
// where it is used, forward and backward, and never stored.
//
//   key(r) = the 64-bit mixer of (seed + step * kStepStride, r);  kept iff draw24((k0 + c) C1, k1) >= T = p 2^24 rounded
//   y = x 2^24 / (2^24 - T) where kept, 0 elsewhere (+ residual)
#pragma once

#include "nuq_device.hpp"
#include "nuq_layer_norm_kernels.hpp"

namespace nuq {

// What a step's number is multiplied with before it is added to the seed: odd, so that no two steps share a seed.
constexpr uint64_t kStepStride = 0xD1342543DE82EF95ull;

struct Draws {
    uint64_t seed;
    const int64_t *step;        // device, may be none: 0
    uint32_t threshold;         // of 2^24
    float keep;                 // 2^24 / (2^24 - threshold), 0 where nothing is kept
    __device__ __forceinline__ uint64_t begin() const { return seed + (step ? (uint64_t)*step * kStepStride : 0ull); }
};

// x[e] <- 0 where element at + e of the row whose key this is is dropped, whatever it was.  (u >= T for the upper 24 bits u of a word is
// word >= 2^8 T, whatever the other bits; T = 2^24 drops all.)
template <int N>
__device__ __forceinline__ void drop(float (&x)[N], BucketKey key, uint32_t at, uint32_t threshold)
{
    const uint32_t first = (key.k0 + at) * kRngC1, least = threshold << 8;
    if (threshold >> 24) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            x[e] = 0.0f;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const uint32_t y = first + (uint32_t)e * kRngC1;
            uint32_t word = __builtin_amdgcn_bitop3_b32(y, y >> 15, key.k1, 0x96) * kRngC2;      // draw24, before its last shift
            word ^= word >> 16;
            x[e] = word >= least ? x[e] : 0.0f;
        }
    }
}

struct Dropout {
    const void *x, *residual;                  // residual: may be none
    void *y;
    Draws draws;
    uint64_t rows, ldx, ldr, ldy;              // row strides in elements
    uint32_t hidden;
};

// A vector of 16 bytes at a time per thread, the launch's vectors one after the other over the rows; the next one's place follows
// from the present one's without a division.  The key is a few 64-bit products per vector, the draw of an element two 32-bit
// products beside six other instructions.  Bound by HBM: 16384 rows of 6400 in bfloat16 with a residual take 102 us, 6.2 TB/s; 5003 of 1001 in fp32
// 8.0 us (8.5 in a trace), two of them the launch.  128 rows of 1600, which the launch bounds: 2.7 us.  (kOnce: the first of these took 107 us without.)
template <class T, bool kResidual, bool kOnce>
__global__ __launch_bounds__(256) void k_dropout(const Dropout P)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    const uint32_t per = (P.hidden + VEC - 1) / VEC, all = gridDim.x * 256u;        // (a launch has fewer than 2^32 threads)
    const uint32_t rows_on = all / per, on = all % per;
    uint32_t v = blockIdx.x * 256u + threadIdx.x;
    uint64_t row = v / per;
    v %= per;
    const uint64_t begin = P.draws.begin();
    for (; row < P.rows; row += rows_on) {
        const uint32_t at = v * VEC;
        const int64_t have = (int64_t)P.hidden - at;
        float x[VEC], r[VEC];
        load_some<VEC, false, kOnce>(x, static_cast<const T *>(P.x) + row * P.ldx + at, have);
        if constexpr (kResidual)
            load_some<VEC, false, kOnce>(r, static_cast<const T *>(P.residual) + row * P.ldr + at, have);
        if (P.draws.threshold) {
            drop<VEC>(x, bucket_key(begin, row), at, P.draws.threshold);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                x[e] *= P.draws.keep;
        }
        if constexpr (kResidual)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                x[e] += r[e];
        store_some<VEC, false, kOnce>(static_cast<T *>(P.y) + row * P.ldy + at, x, have);
        v += on;
        if (v >= per) {
            v -= per;
            ++row;
        }
    }
}

}  // namespace nuq
