// Device code that the optimizer's and the layer norm's kernels share: element types and their vectors, sums and maxima over
// lanes, and the table of tensors that a launch over many of them carries in its arguments.
#pragma once

#include <cstdint>
#include <hip/hip_runtime.h>

namespace nuq {

// N elements at any address that is a multiple of the element: global memory takes 16 bytes from there at once.
template <class T, int N>
struct VecOf {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <class T, int N>
using Vec = typename VecOf<T, N>::type;

// kOnce: with the hint that the memory is touched once.
template <int N, bool kOnce = false, class T>
__device__ __forceinline__ void load_as_float(float (&to)[N], const T *from)
{
    Vec<T, N> v;
    if constexpr (kOnce)
        v = __builtin_nontemporal_load(reinterpret_cast<const Vec<T, N> *>(from));
    else
        v = *reinterpret_cast<const Vec<T, N> *>(from);
#pragma unroll
    for (int e = 0; e < N; ++e)
        to[e] = (float)v[e];
}

// Rounded to the nearest T, ties to even.
template <int N, bool kOnce = false, class T>
__device__ __forceinline__ void store_from_float(T *to, const float (&from)[N])
{
    Vec<T, N> v;
#pragma unroll
    for (int e = 0; e < N; ++e)
        v[e] = (T)from[e];
    if constexpr (kOnce)
        __builtin_nontemporal_store(v, reinterpret_cast<Vec<T, N> *>(to));
    else
        *reinterpret_cast<Vec<T, N> *>(to) = v;
}

// The same for the first `have` elements; the others read as 0 and are not written.  kWhole: there are N.
template <int N, bool kWhole = false, bool kOnce = false, class T>
__device__ __forceinline__ void load_some(float (&to)[N], const T *from, int64_t have)
{
    if (kWhole || have >= N) {
        load_as_float<N, kOnce>(to, from);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            to[e] = e < have ? (float)from[e] : 0.0f;
    }
}
template <int N, bool kWhole = false, bool kOnce = false, class T>
__device__ __forceinline__ void store_some(T *to, const float (&from)[N], int64_t have)
{
    if (kWhole || have >= N) {
        store_from_float<N, kOnce>(to, from);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < have)
                to[e] = (T)from[e];
    }
}

template <int kCtrl>
__device__ __forceinline__ float dpp_move(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kCtrl, 0xf, 0xf, true));
}

// Sum over teams of TEAM neighbouring lanes, the same bits in each of them: every step adds two disjoint groups, and a + b is
// b + a.
template <int TEAM>
__device__ __forceinline__ float team_sum(float x)
{
    static_assert(TEAM == 4 || TEAM == 16 || TEAM == 32 || TEAM == 64, "team");
    x += dpp_move<0xB1>(x);             // lane ^ 1
    x += dpp_move<0x4E>(x);             // lane ^ 2
    if constexpr (TEAM >= 16) {
        x += dpp_move<0x141>(x);        // 7 - lane of each eight
        x += dpp_move<0x140>(x);        // 15 - lane of each sixteen
    }
    if constexpr (TEAM >= 32) {         // the sums of sixteen, read out of one lane of each
        const auto of = [&](int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane)); };
        const float low = of(0) + of(16), high = of(32) + of(48);
        x = TEAM == 64 ? low + high : threadIdx.x % 64u < 32u ? low : high;
    }
    return x;
}

// Maximum of whole numbers over the wave, the same in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true));    // row_shr:1
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true));    // row_shr:2
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true));    // row_shr:4
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true));    // row_shr:8
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, true));    // row_bcast:15
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, true));    // row_bcast:31
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// Sum of doubles over a workgroup of WG threads, in a fixed order; valid in thread 0.  red: WG / 64 doubles of LDS.
template <int WG>
__device__ __forceinline__ double workgroup_sum(double x, double *red)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        x += __shfl_down(x, off, 64);
    if (threadIdx.x % 64u == 0)
        red[threadIdx.x / 64u] = x;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int k = 1; k < WG / 64; ++k)
            x += red[k];
    return x;
}

// Tensors per launch: a wave looks at one entry per lane, and the tables of all their arrays fit the 4 KiB of a launch's
// arguments.
constexpr uint32_t kTableTensors = 64;

// start[i]: the first chunk of tensor i, 2^32 - 1 where there is none.  The tensor that `chunk` belongs to: one load for all.
template <uint32_t kTensors>
__device__ __forceinline__ uint32_t tensor_of(const uint32_t (&start)[kTensors], uint32_t chunk)
{
    static_assert(kTensors <= 64, "a tensor per lane");
    const uint32_t lane = threadIdx.x % 64u, begin = lane < kTensors ? start[lane] : ~0u;
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)__popcll(__ballot(begin <= chunk)) - 1);
}

}  // namespace nuq
