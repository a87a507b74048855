// Tiles of a matrix product on the matrix cores: acc[m][n] = sum over k of A[m][k] B[n][k].
//
// A workgroup of WM x WN waves has a tile of BM x BN; a wave BM / WM x BN / WN of it in 16 x 16 blocks.  Per step a depth of 128 bytes
// (64 elements of 16 bits, 32 of fp32) goes from global memory into one of the stages in the LDS, without a register between, while the
// products of another run; operands come out of the LDS half a step ahead of their products, also over a step's end, and the order of reads,
// loads and products is fixed.  Two stages for tiles whose products take longer than a load; four for tiles of few rows, which only pass
// the other operand by.  The loads write the LDS in lane order, so where banks would be met twice it is the address in global memory that
// is permuted.
//
// The matrix cores bound a large tile, at the clock that their power leaves: 16 x 16 x 32 moves half of the accumulators that 32 x 32 x 16
// does.  8192 x 8192 x 8192 in bfloat16: 1351 TFLOP/s, cores busy for 0.69 of the cycles at 2.0 GHz; with 32 x 32 x 16 1336, 0.80 at
// 1.67 GHz; and 1274 with reads that begin with the step.  (A library product reaches 1630 there.)
//
// An operand stands in memory by rows, k contiguous: in the LDS 128 bytes of each, chunk c (16 bytes) of row r at c ^ r / 2 % 8.  Sixteen
// lanes read a column of chunks at once, two rows fill the 64 banks, and so these meet each bank once.  Or it stands across, m or n
// contiguous: in the LDS the rows of k, and elements of 16 bits are transposed by the reads, 4 x 16 of them at a time: 32 lanes read 32
// bytes of rows k to k + 3 and k + 8 to k + 11, of which piece c (32 bytes) is at c ^ (k % 4 * 2 + k / 8 % 2); fp32 is read element by
// element, 64 bytes of rows k, k + 4, k + 8 and k + 12, of which piece c (64 bytes) is at c ^ k / 4 % 4.
//
// fp32 operands go through the matrix cores as fp32: a chunk is four products of depth 4, and which k a lane holds is the same in
// both operands, so the sum is over every k once.
#pragma once

#include <cstdint>
#include <hip/hip_runtime.h>

namespace nuq {

typedef float Block __attribute__((ext_vector_type(4)));    // lane l, register r: m = 4 (l / 16) + r, n = l % 16
typedef uint32_t Chunk __attribute__((ext_vector_type(4)));  // 16 bytes of a row: of lane l those behind 16 (l / 16) bytes of k

template <class T>
__device__ __forceinline__ Block multiply(Chunk a, Chunk b, Block c)
{
    if constexpr (sizeof(T) == 4) {
        typedef float F4 __attribute__((ext_vector_type(4)));
        const F4 x = __builtin_bit_cast(F4, a), y = __builtin_bit_cast(F4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
        return c;
    } else {
        typedef T T8 __attribute__((ext_vector_type(8)));
        const T8 x = __builtin_bit_cast(T8, a), y = __builtin_bit_cast(T8, b);
        if constexpr (__is_same(T, __bf16))
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
    }
}

// 4 x 16 elements of 16 bits out of the LDS: lane l of sixteen brings the address of elements 4 (l % 4) to 4 (l % 4) + 3 of row l / 4 and
// gets element l of the four rows.
typedef uint32_t HalfChunk __attribute__((ext_vector_type(2)));
__device__ __forceinline__ HalfChunk read_transposed(const char *at)
{
#ifdef __HIP_DEVICE_COMPILE__                                // (the host's pass does not know the builtin)
    typedef short S4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(HalfChunk, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4 *)at));
#else
    return HalfChunk{};
#endif
}

// 16 bytes per lane from buffer + at + offset into the LDS, one lane's behind the other's; zeros for what lies behind the buffer.
__device__ __forceinline__ void load_into_lds(__amdgpu_buffer_rsrc_t buffer, char *to, uint32_t at, uint32_t offset)
{
#ifdef __HIP_DEVICE_COMPILE__                                // (nor that this one takes 16 bytes)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (__attribute__((address_space(3))) void *)to, 16, at, offset, 0, 0);
#endif
}

// The thread's place in its workgroup, or lane, where what follows from it is reckoned again for every tile: kept from one tile to the
// next it would fill the registers that the products need.
__device__ __forceinline__ uint32_t thread_again()
{
    uint32_t t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}
__device__ __forceinline__ uint32_t lane_again() { return thread_again() % 64u; }

// All that the workgroup's waves had of the LDS is read and written behind this, loads from global memory may still be on their way.  (The
// builtins touch no memory as far as the compiler knows: the clobbers keep accesses on their side.)
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);                      // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A tile's operand.  By rows: the tile's first row, the bytes from one to the next, how many there are, the chunks of each.  Across: the
// tile's first column in the first row of k, the bytes from one k to the next, the chunks of each, how many k there are.  Addresses and
// strides are multiples of 16, a stride is below 2^22.
struct Operand {
    const void *first;
    uint32_t stride, wide, deep;
};

// An offset that no buffer of a tile reaches (fewer than 2^31 bytes each): the load brings 0.
constexpr uint32_t kNowhere = 0x80000000u;

// One operand's part of a stage, SIZE rows or columns of it, loaded by WAVES waves.
template <class T, int SIZE, int WAVES, bool kAcross>
struct OperandLoads {
    static constexpr int LOADS = SIZE / 8 / WAVES;           // per wave and step, 1024 bytes each
    static constexpr uint32_t DEPTH = 128 / sizeof(T);       // of a step
    static constexpr uint32_t ROW = kAcross ? SIZE * (uint32_t)sizeof(T) : 128u;            // bytes of a row in the LDS
    static constexpr int READS = !kAcross ? 1 : sizeof(T) == 2 ? 2 : 4;                     // of the LDS per block and half step
    static_assert(LOADS * 8 * WAVES == SIZE && WAVES % 2 == 0, "whole loads");
    static_assert(!kAcross || (1024u % ROW == 0 && ROW / 16u >= 16u), "whole rows, and what is permuted in them");

    Operand O;
    uint32_t at[LOADS];                                      // offsets of the lane's chunks in a step
    uint32_t chunk;                                          // by rows: the lane's chunk in every row that it loads

    __device__ __forceinline__ void place(const Operand &o, uint32_t wave, uint32_t lane)
    {
        O = o;
        chunk = lane % 8u ^ (wave % 2u * 4u + lane / 16u);   // (a load is of rows 8 g to 8 g + 7, g odd in odd waves)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t byte = ((uint32_t)i * WAVES + wave) * 1024u + lane * 16u, row = byte / ROW;
            if constexpr (kAcross) {
                const uint32_t c = byte % ROW / 16u, turn = sizeof(T) == 2 ? row % 4u * 4u + row / 8u % 2u * 2u : row / 4u % 4u * 4u, column = c ^ turn;
                at[i] = column < O.wide ? row * O.stride + column * 16u : kNowhere;
            } else {
                at[i] = row < O.wide ? row * O.stride + chunk * 16u : kNowhere;
            }
        }
    }
    // The loads of step s.
    __device__ __forceinline__ void issue(uint32_t s, char *__restrict__ to, uint32_t wave) const
    {
        const char *first = static_cast<const char *>(O.first);
        uint32_t rows = O.wide, offset = s * 128u;
        bool there = chunk + s * 8u < O.deep;
        if constexpr (kAcross) {
            first += (uint64_t)(s * DEPTH) * O.stride;
            rows = s * DEPTH < O.deep ? min(DEPTH, O.deep - s * DEPTH) : 0u;
            offset = 0;
            there = true;
        }
        const auto buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(first), 0, (int)(rows * O.stride), 0x00020000);
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            load_into_lds(buffer, to + ((uint32_t)i * WAVES + wave) * 1024u, there ? at[i] : kNowhere, offset);
    }
    // Where a lane reads: its place in the blocks of 16 rows or columns from `begin` on (a multiple of all that the wave has), and the
    // operands of a half step from there.
    static __device__ __forceinline__ uint32_t place_of(uint32_t begin, uint32_t lane)
    {
        if constexpr (!kAcross) {
            return (begin + lane % 16u) * 128u + (lane / 16u ^ lane / 2u % 8u) * 16u;
        } else if constexpr (sizeof(T) == 2) {               // four columns of row k % 4 = lane / 4 % 4
            const uint32_t k = lane / 16u * 8u + lane / 4u % 4u;
            return k * ROW + (begin / 16u ^ (k % 4u * 2u + k / 8u % 2u)) * 32u + lane % 4u * 8u;
        } else {
            return lane / 16u * 4u * ROW + (begin / 16u ^ lane / 16u) * 64u + lane % 16u * 4u;
        }
    }
    template <int N>
    static __device__ __forceinline__ void read(Chunk (&to)[N], const char *__restrict__ from, uint32_t place, int half)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (!kAcross) {
                to[i] = *reinterpret_cast<const Chunk *>(from + (place ^ (uint32_t)half * 64u) + i * 2048);
            } else if constexpr (sizeof(T) == 2) {
                const char *const at = from + (place ^ (uint32_t)i * 32u) + half * 32 * (int)ROW;
                const HalfChunk low = read_transposed(at), high = read_transposed(at + 4 * ROW);
                to[i] = Chunk{low[0], low[1], high[0], high[1]};
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    to[i][e] = *reinterpret_cast<const uint32_t *>(from + (place ^ (uint32_t)i * 64u) + (half * 16 + e) * (int)ROW);
            }
        }
    }
};

template <class T, int BM_, int BN_, int WM_, int WN_, int STAGES_, bool kAcrossA = false, bool kAcrossB = false>
struct ProductTile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;             // blocks of a wave
    static constexpr int STAGES = STAGES_, STAGE = (BM + BN) * 128, LDS = STAGES * STAGE;
    using LoadsA = OperandLoads<T, BM, WAVES, kAcrossA>;
    using LoadsB = OperandLoads<T, BN, WAVES, kAcrossB>;

    Block acc[MI][NI];

    __device__ __forceinline__ explicit ProductTile(char *lds_) : lds(lds_), last(STAGES - 1u)
    {
        const uint32_t lane = threadIdx.x % 64u;
        wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
        place_a = LoadsA::place_of(wave / WN * (BM / WM), lane);
        place_b = BM * 128u + LoadsB::place_of(wave % WN * (BN / WN), lane);
    }
    // The tile whose products come next, of `steps` steps (there are two at least, of zeros if need be): its first ones go into the stages
    // behind the last that is read.
    __device__ __forceinline__ void begin(const Operand &A, const Operand &B, uint32_t steps_)
    {
        const uint32_t lane = lane_again();
        steps = max(steps_, 2u);
        a.place(A, wave, lane);
        b.place(B, wave, lane);
#pragma unroll
        for (uint32_t s = 0; s < STAGES - 1u; ++s)
            if (s < steps) {
                char *const to = stage(last + 1u + s);
                a.issue(s, to, wave);
                b.issue(s, to + BM * 128, wave);
            }
    }
    // Its products but those of the last step, which finish() brings.  Between the two is the place of begin() for the tile after it: that
    // tile's first loads are on their way while this one's results are written.
    __device__ __forceinline__ void run()
    {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
                acc[i][j] = Block{};
        arrive(0u);
        last = wrap(last + 1u);
        LoadsB::read(y[0], stage(last), place_b, 0);
        LoadsA::read(x[0], stage(last), place_a, 0);
        if (STAGES - 1u < steps)
            issue(STAGES - 1u, stage(last + STAGES - 1u));
        __builtin_amdgcn_sched_barrier(0);
        uint32_t s = 0;
        for (; s + STAGES < steps; ++s)
            step<true, true>(s);
        if constexpr (STAGES > 2)
            for (; s + 2u < steps; ++s)
                step<true, false>(s);
        step<false, false>(s);
    }
    // (Nothing is read ahead here: begin() and what the caller has for the results take registers too.)
    __device__ __forceinline__ void finish()
    {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            LoadsB::read(y[half], stage(last), place_b, half);
            LoadsA::read(x[half], stage(last), place_a, half);
            half_step<false, false>(half, nullptr, nullptr, 0u);
        }
    }

    // The stage read last, for the waves' own use behind finish(): until the next run().  All waves call it.
    __device__ __forceinline__ char *free_stage() const
    {
        lds_barrier();                                       // (the others may still read it)
        return stage(last);
    }

    // Rows n of results in 16 bits by way of the stage read last, so that 16 bytes of a lane and whole lines of a wave are written: call
    // behind finish(), from all waves.  value(j, i, x): x[e] of column 4 (lane / 16) + e of block i, row lane % 16 of block j.
    // to(j, row): where the wave's columns of that row are, none for a row that is not there; `have` of them are.
    template <class V, class P>
    __device__ __forceinline__ void store_rows(V &&value, P &&to, int64_t have)
    {
        static_assert(sizeof(T) == 2, "16 bits");
        constexpr uint32_t CHUNKS = MI * 2, PER = 64 / CHUNKS;            // of a row; rows per instruction
        static_assert(WAVES * 16 * CHUNKS * 16 <= STAGE && PER <= 16, "a wave's rows");
        const uint32_t lane = lane_again(), row = lane % 16u;
        const auto turn = [](uint32_t r) { return r / (16u / CHUNKS) % CHUNKS; };                // (as the operands': no bank twice)
        char *const own = free_stage() + wave * (16u * CHUNKS * 16u);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                typedef T T4 __attribute__((ext_vector_type(4)));
                float x[4];
                value(j, i, x);
                *reinterpret_cast<T4 *>(own + row * (CHUNKS * 16u) + ((i * 2u + lane / 32u) ^ turn(row)) * 16u + lane / 16u % 2u * 8u) =
                    T4{(T)x[0], (T)x[1], (T)x[2], (T)x[3]};
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (uint32_t k = 0; k < 16u / PER; ++k) {
                const uint32_t r = k * PER + lane / CHUNKS, c = lane % CHUNKS;
                const Chunk chunk = *reinterpret_cast<const Chunk *>(own + r * (CHUNKS * 16u) + (c ^ turn(r)) * 16u);
                T *const at = to(j, r);
                if (at) {
                    typedef T T8 __attribute__((ext_vector_type(8), aligned(sizeof(T))));
                    const T8 x = __builtin_bit_cast(T8, chunk);
                    const int64_t left = have - (int64_t)c * 8;
                    if (left >= 8) {
                        *reinterpret_cast<T8 *>(at + c * 8u) = x;
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (e < left)
                                at[c * 8u + e] = x[e];
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
    // The wave's first column and row in the tile.
    __device__ __forceinline__ uint32_t first_m() const { return wave / WN * (BM / WM); }
    __device__ __forceinline__ uint32_t first_n() const { return wave % WN * (BN / WN); }

private:
    char *const lds;
    LoadsA a;
    LoadsB b;
    uint32_t wave, steps, last, place_a, place_b;            // last: the stage that is read, or was last
    Chunk x[2][MI], y[2][NI];                                // operands of the half step whose products run, and of the next one

    // k below 2 STAGES.
    static __device__ __forceinline__ uint32_t wrap(uint32_t k) { return STAGES == 3 ? (k >= 3u ? k - 3u : k) : k % STAGES; }
    __device__ __forceinline__ char *stage(uint32_t k) const { return lds + wrap(k) * STAGE; }

    // Step s's loads of all waves are in the LDS, and all reads of the stage before it are done.  (By the builtin, not inline asm: what else
    // was loaded before is there too, and the compiler knows.)
    __device__ __forceinline__ void arrive(uint32_t s) const
    {
        constexpr int EACH = LoadsA::LOADS + LoadsB::LOADS;  // loads of a step, which later steps may leave on their way
        const uint32_t later = min(STAGES - 2u, steps - 1u - s);
        asm volatile("" ::: "memory");
        if (STAGES >= 4 && later == 2u)
            __builtin_amdgcn_s_waitcnt(counter(2 * EACH));
        else if (STAGES >= 3 && later == 1u)
            __builtin_amdgcn_s_waitcnt(counter(EACH));
        else
            __builtin_amdgcn_s_waitcnt(counter(0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
    static constexpr int counter(int loads) { return 0x0070 | (loads & 15) | loads >> 4 << 14; }      // vmcnt(loads) lgkmcnt(0)
    static_assert(STAGES >= 2 && STAGES <= 4 && (STAGES - 2) * (LoadsA::LOADS + LoadsB::LOADS) < 64, "what is counted");

    __device__ __forceinline__ void issue(uint32_t s, char *__restrict__ to) const
    {
        a.issue(s, to, wave);
        b.issue(s, to + BM * 128, wave);
    }
    // The products of step s, which is not the last.  Behind its first half all waves have read what they need of its stage, and the next
    // one's loads are there: with kRead operands of the next come from there, and with kLoad its own stage takes the loads of step s + STAGES.
    template <bool kRead, bool kLoad>
    __device__ __forceinline__ void step(uint32_t s)
    {
        half_step<true, false>(0, stage(last), nullptr, 0u);
        arrive(s + 1u);
        last = wrap(last + 1u);
        half_step<kRead, kLoad>(1, stage(last), stage(last + STAGES - 1u), s + STAGES);
    }
    // The products of half `half` of a step, with the reads of the half after it from the stage `from` and the loads of step `next` into the
    // stage `to`.  (That the two do not overlap has to be said: reads of the LDS would wait for the loads otherwise.  The order is fixed:
    // reads over the first three quarters of the products, loads over the first half: 1351 TFLOP/s instead of 1333 over all of them, and
    // gradients of 8192 x 1600 against 50257 in 3360 us instead of 3513; in fp32 it is the same to 1 %.)
    template <bool kRead, bool kLoad>
    __device__ __forceinline__ void half_step(int half, const char *__restrict__ from, char *__restrict__ to, uint32_t next)
    {
        constexpr int PRODUCTS = MI * NI * (sizeof(T) == 4 ? 4 : 1), READS = kRead ? MI * LoadsA::READS + NI * LoadsB::READS : 0;
        constexpr int LOADS = kLoad ? LoadsA::LOADS + LoadsB::LOADS : 0;
        if constexpr (kRead) {
            LoadsB::read(y[half ^ 1], from, place_b, half ^ 1);
            LoadsA::read(x[half ^ 1], from, place_a, half ^ 1);
        }
        if constexpr (kLoad)
            issue(next, to);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
                acc[i][j] = multiply<T>(x[half][i], y[half][j], acc[i][j]);
        constexpr int PER_READ = READS * 4 <= PRODUCTS * 3 && READS > 0 ? PRODUCTS * 3 / 4 / READS : 1;
        constexpr int PER_LOAD = LOADS > 0 && LOADS * 2 <= PRODUCTS ? PRODUCTS / 2 / LOADS : 1;
#pragma unroll
        for (int k = 0; k < PRODUCTS; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);             // a product
            if (READS > 0 && k % PER_READ == PER_READ - 1)
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);         // a read of the LDS
            if (LOADS > 0 && k % PER_LOAD == 0 && k / PER_LOAD < LOADS)
                __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);         // a load
        }
        __builtin_amdgcn_sched_barrier(0);
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
