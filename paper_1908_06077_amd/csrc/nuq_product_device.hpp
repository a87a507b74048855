// Tiles of a matrix product on the matrix cores: acc[m][n] = sum over k of A[m][k] B[n][k], both operands with k contiguous.
//
// A workgroup of WM x WN waves has a tile of BM x BN; a wave BM / WM x BN / WN of it in 32 x 32 blocks.  Per step 128 bytes of every
// row (64 elements of 16 bits, 32 of fp32) go from global memory into one half of the LDS, without a register between, while the
// products of the other half run; operands come out of the LDS one quarter step ahead of their products.  In the LDS chunk c (16
// bytes) of row r stands at c ^ r % 8: the eight lanes that read one column of chunks at once meet eight different groups of banks.
// The loads write the LDS in lane order, so it is the address in global memory that is permuted.
//
// fp32 operands go through the matrix cores as fp32: a chunk is four products of depth 2, and which k a lane holds is the same in
// both operands, so the sum is over every k once.
#pragma once

#include <cstdint>
#include <hip/hip_runtime.h>

namespace nuq {

typedef float Block __attribute__((ext_vector_type(16)));   // lane l, register r: m = 8 (r / 4) + 4 (l / 32) + r % 4, n = l % 32
typedef uint32_t Chunk __attribute__((ext_vector_type(4)));  // 16 bytes of a row

template <class T>
__device__ __forceinline__ Block multiply(Chunk a, Chunk b, Block c)
{
    if constexpr (sizeof(T) == 4) {
        typedef float F4 __attribute__((ext_vector_type(4)));
        const F4 x = __builtin_bit_cast(F4, a), y = __builtin_bit_cast(F4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], c, 0, 0, 0);
        return c;
    } else {
        typedef T T8 __attribute__((ext_vector_type(8)));
        const T8 x = __builtin_bit_cast(T8, a), y = __builtin_bit_cast(T8, b);
        if constexpr (__is_same(T, __bf16))
            return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0);
    }
}

// Rows of a tile: the first one's address, the bytes from one to the next (a multiple of 16), and how many there are.
struct TileRows {
    const void *first;
    uint32_t stride, there;
};

// An offset that no buffer of a tile reaches (fewer than 2^31 bytes each): the load brings 0.
constexpr uint32_t kNowhere = 0x80000000u;

template <class T, int BM_, int BN_, int WM_, int WN_>
struct ProductTile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int MI = BM / WM / 32, NI = BN / WN / 32;             // blocks of a wave
    static constexpr int STAGE = (BM + BN) * 128, LDS = 2 * STAGE;
    static constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;         // loads per wave and step, of eight rows each
    static_assert(LA * 8 * WAVES == BM && LB * 8 * WAVES == BN, "whole loads");

    Block acc[MI][NI];

    // chunks: of 16 bytes per row, the operands' depth; what lies behind them in a row is not read.
    __device__ __forceinline__ void run(const TileRows &A, const TileRows &B, uint32_t chunks, char *lds)
    {
        const uint32_t lane = threadIdx.x % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
        Loads L{__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(A.first), 0, (int)(A.there * A.stride), 0x00020000),
                __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(B.first), 0, (int)(B.there * B.stride), 0x00020000),
                {}, {}, lane % 8u ^ lane / 8u, wave};
        places(L.a, A, L.chunk, wave, lane);
        places(L.b, B, L.chunk, wave, lane);
        const uint32_t swizzled = (lane / 32u ^ lane % 8u) * 16u;
        const uint32_t a = (wave / WN * (BM / WM) + lane % 32u) * 128u + swizzled;
        const uint32_t b = BM * 128u + (wave % WN * (BN / WN) + lane % 32u) * 128u + swizzled;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
                acc[i][j] = Block{};
        const uint32_t steps = (chunks + 7u) / 8u;
        if (steps == 0)
            return;
#pragma unroll
        for (int quarter = 0; quarter < 4; ++quarter)
            issue(L, quarter, 0u, chunks, lds);
        uint32_t s = 0;
        for (; s + 1u < steps; ++s) {
            arrive();
            step<true>(lds + s % 2u * STAGE, lds + (s + 1u) % 2u * STAGE, a, b, L, s + 1u, chunks);
        }
        arrive();
        step<false>(lds + s % 2u * STAGE, lds, a, b, L, 0u, 0u);
        __syncthreads();                                     // (the LDS is free for what follows)
    }

private:
    struct Loads {
        __amdgpu_buffer_rsrc_t ra, rb;
        uint32_t a[LA], b[LB];                               // offsets of the lane's chunks at depth 0
        uint32_t chunk, wave;                                // the lane's chunk in every row that it loads
    };
    template <int N>
    static __device__ __forceinline__ void places(uint32_t (&to)[N], const TileRows &R, uint32_t chunk, uint32_t wave, uint32_t lane)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t row = ((uint32_t)i * WAVES + wave) * 8u + lane / 8u;
            to[i] = row < R.there ? row * R.stride + chunk * 16u : kNowhere;
        }
    }
    // The loads of one quarter of step s.
    static __device__ __forceinline__ void issue(const Loads &L, int quarter, uint32_t s, uint32_t chunks, char *__restrict__ to)
    {
        using Lds = __attribute__((address_space(3))) void *;
        const bool there = L.chunk + s * 8u < chunks;
#pragma unroll
        for (int i = quarter * (LA + LB) / 4; i < (quarter + 1) * (LA + LB) / 4; ++i) {
            if (i < LA)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(L.ra, (Lds)(to + (i * WAVES + L.wave) * 1024u), 16, there ? L.a[i < LA ? i : 0] : kNowhere,
                                                         s * 128u, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(L.rb, (Lds)(to + BM * 128 + ((i - LA) * WAVES + L.wave) * 1024u), 16,
                                                         there ? L.b[i < LA ? 0 : i - LA] : kNowhere, s * 128u, 0, 0);
        }
    }
    // All loads of all waves are in the LDS, and all reads of the other half are done.
    static __device__ __forceinline__ void arrive()
    {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    static __device__ __forceinline__ void operands(Chunk (&x)[MI], Chunk (&y)[NI], const char *__restrict__ from, uint32_t a, uint32_t b,
                                                    int quarter)
    {
#pragma unroll
        for (int i = 0; i < MI; ++i)
            x[i] = *reinterpret_cast<const Chunk *>(from + (a ^ (uint32_t)quarter * 32u) + i * 4096);
#pragma unroll
        for (int j = 0; j < NI; ++j)
            y[j] = *reinterpret_cast<const Chunk *>(from + (b ^ (uint32_t)quarter * 32u) + j * 4096);
    }
    // The products of the half `from`; the loads of step `next` into the half `to`.  (That the two do not overlap has to be said: reads
    // of the LDS would wait for the loads otherwise.  The order is fixed: left to itself the compiler asks for the loads last.)
    template <bool kLoad>
    __device__ __forceinline__ void step(const char *__restrict__ from, char *__restrict__ to, uint32_t a, uint32_t b, const Loads &L,
                                         uint32_t next, uint32_t chunks)
    {
        Chunk x[2][MI], y[2][NI];
        operands(x[0], y[0], from, a, b, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int quarter = 0; quarter < 4; ++quarter) {
            if (quarter < 3)
                operands(x[(quarter + 1) & 1], y[(quarter + 1) & 1], from, a, b, quarter + 1);
            if (kLoad && quarter < 2) {                      // (early, so that they have the step to arrive)
                issue(L, 2 * quarter, next, chunks, to);
                issue(L, 2 * quarter + 1, next, chunks, to);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
                    acc[i][j] = multiply<T>(x[quarter & 1][i], y[quarter & 1][j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// Which tile of `mt` x `nt` a workgroup has.  The XCDs take workgroups in turn, and each has an L2 of its own: an XCD's workgroups are
// neighbours, in bands of eight tiles of n.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t mt, uint32_t nt, uint32_t &m, uint32_t &n)
{
    const uint32_t all = mt * nt, each = all / 8u, more = all % 8u, xcd = id % 8u;
    id = xcd * each + min(xcd, more) + id / 8u;              // (the first `more` XCDs have one more)
    const uint32_t band = id / (8u * mt), within = id % (8u * mt), wide = min(8u, nt - band * 8u);
    n = band * 8u + within % wide;
    m = within / wide;
}

}  // namespace nuq
