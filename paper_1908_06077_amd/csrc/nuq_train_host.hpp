// Host code of the operators of transformer training: element types, checks of arrays, and what a launch may have.
#pragma once

#include <atomic>
#include <cstdint>

#include "nuq_host.hpp"

namespace nuq {

template <class T>
struct Type {
    using type = T;
};

// f(Type<element>) for one of the three element types.
template <class F>
int with_type(uint32_t type, F &&f)
{
    return type == NUQ_F32 ? f(Type<float>{}) : type == NUQ_BF16 ? f(Type<__bf16>{}) : f(Type<_Float16>{});
}

inline uint32_t width(uint32_t type) { return type == NUQ_F32 ? 4u : 2u; }

inline bool off_grid(const void *p, uint32_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1u)) != 0; }

inline bool valid_array(const void *p, uint64_t n, uint32_t bytes) { return n == 0 || (p && !off_grid(p, bytes)); }

// Whether results stand where the rows they are of stood, but at another stride: rows that are not read yet would be overwritten.
inline bool other_stride(const void *to, uint64_t ld, const void *of, uint64_t ld_of) { return to && to == of && ld != ld_of; }

// Arrays that fit this are read and written plainly: they may still be there, and stay for what comes next.  Larger ones take
// non-temporal loads and stores: an AdamW step on 25.6 M elements (409 MB) 163 -> 130 us, on 1.56 G 8.10 -> 7.52 ms; on 117 MB
// of 8-bit states, weights and gradients they cost 2 %.  Between (134 to 300 MB) they win 5 % where the arrays have left the cache
// and lose 20 % where they have not.
constexpr uint64_t kLastLevelCache = 256ull << 20;

// Workgroups of 256 threads that a launch has at most: it has fewer than 2^32 threads.
constexpr uint64_t kMostGroups = 1ull << 23;
static_assert(kMostGroups * 256u < 1ull << 32, "threads of a launch");

// Workgroups of `threads` threads of a kernel that the current device holds at once (0 on error), looked up once per kernel and
// device.
template <auto kernel>
uint32_t resident_workgroups(uint32_t threads)
{
    static std::atomic<uint32_t> known[64];
    int dev = 0, per_cu = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0)
        return 0;
    uint32_t have = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0u;
    if (!have) {
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, reinterpret_cast<const void *>(kernel), (int)threads, 0) != hipSuccess ||
            hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || per_cu < 1 || cus < 1)
            return 0;
        have = (uint32_t)per_cu * (uint32_t)cus;
        if (dev < 64)
            known[dev].store(have, std::memory_order_relaxed);
    }
    return have;
}

// f(Type<element>, Type<weight>)
template <class F>
int with_types(uint32_t type, uint32_t weight_type, F &&f)
{
    return with_type(type, [&](auto t) { return weight_type == type ? f(t, t) : f(t, Type<float>{}); });
}

}  // namespace nuq
