// AdamW over many tensors in one launch, with states in 32 bits or in 8, and the norm of all gradients with the factor that
// clips them.
//
//   g = c * gradient;  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   w <- w (1 - alpha lambda) - alpha / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// m and v are evaluated in fp32, every product and every sum rounded (the 8-bit codes have to come out the same wherever they
// are computed); w takes a hardware square root and reciprocal (1 unit of the last place each) on a term that is a thousandth
// of the weight, and fused multiply-adds.
#pragma once

#include "nuq_train_device.hpp"

namespace nuq {

struct AdamwNumbers {
    float b1, c1, b2, c2;   // beta1, 1 - beta1, beta2, 1 - beta2
    float step;             // alpha / (1 - beta1^t)
    float root;             // 1 / sqrt(1 - beta2^t)
    float eps;
};

__device__ __forceinline__ void adamw_moments(float &m, float &v, float g, const AdamwNumbers &N)
{
    m = m * N.b1 + g * N.c1;              // (the file is compiled without contraction)
    v = v * N.b2 + (g * g) * N.c2;
}

__device__ __forceinline__ float adamw_weight(float w, float m, float v, float keep, const AdamwNumbers &N)
{
    const float u = m * __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_amdgcn_sqrtf(v), N.root, N.eps));
    return __builtin_fmaf(-N.step, u, w * keep);
}

constexpr uint32_t kAdamwRows = 2;                              // vectors of four that a thread takes
constexpr uint32_t kAdamwChunk = 256u * 4u * kAdamwRows;        // elements per workgroup

struct AdamwTable {
    float *w[kTableTensors], *m[kTableTensors], *v[kTableTensors];
    const void *g[kTableTensors];
    void *copy[kTableTensors];
    uint64_t n[kTableTensors];
    float keep[kTableTensors];              // 1 - alpha * lambda
    uint32_t start[kTableTensors];
    uint32_t count;
    AdamwNumbers num;
    const float *coefficient;               // c, or none
    uint32_t *flags;
};
static_assert(sizeof(AdamwTable) <= 4096, "a launch's arguments");

// One pass: 28 bytes per element with 32-bit gradients.  An element whose new moments are not finite is left as it is.
template <class G, class C, bool kCopy>
__global__ __launch_bounds__(256) void k_adamw(const AdamwTable P)
{
    const uint32_t t = (uint32_t)__builtin_amdgcn_readfirstlane((int)tensor_of(P.start, P.count, blockIdx.x));
    const uint64_t base = (uint64_t)(blockIdx.x - P.start[t]) * kAdamwChunk, n = P.n[t];
    const float keep = P.keep[t], c = P.coefficient ? *P.coefficient : 1.0f;
    float *const pw = P.w[t], *const pm = P.m[t], *const pv = P.v[t];
    const G *const pg = static_cast<const G *>(P.g[t]);
    float w[kAdamwRows][4], m[kAdamwRows][4], v[kAdamwRows][4], g[kAdamwRows][4];
#pragma unroll
    for (uint32_t r = 0; r < kAdamwRows; ++r) {
        const uint64_t i = base + (r * 256u + threadIdx.x) * 4u;
        const int64_t have = (int64_t)n - (int64_t)i;
        load_some<4>(g[r], pg + i, have);
        load_some<4>(m[r], pm + i, have);
        load_some<4>(v[r], pv + i, have);
        load_some<4>(w[r], pw + i, have);
    }
    bool lost = false;
#pragma unroll
    for (uint32_t r = 0; r < kAdamwRows; ++r) {
        const uint64_t i = base + (r * 256u + threadIdx.x) * 4u;
        const int64_t have = (int64_t)n - (int64_t)i;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float m1 = m[r][e], v1 = v[r][e];
            adamw_moments(m1, v1, g[r][e] * c, P.num);
            const bool fine = __builtin_fabsf(m1) < __builtin_inff() && v1 < __builtin_inff();
            lost |= !fine;
            m[r][e] = fine ? m1 : m[r][e];
            v[r][e] = fine ? v1 : v[r][e];
            w[r][e] = fine ? adamw_weight(w[r][e], m1, v1, keep, P.num) : w[r][e];
        }
        store_some<4>(pm + i, m[r], have);
        store_some<4>(pv + i, v[r], have);
        store_some<4>(pw + i, w[r], have);
        if constexpr (kCopy)
            store_some<4>(static_cast<C *>(P.copy[t]) + i, w[r], have);
    }
    if (__any(lost) && threadIdx.x % 64u == 0)
        atomicOr(P.flags, NUQ_FLAG_NONFINITE);
}

// ---- states in 8 bits ----
// Blocks of 256 elements, one per wave at a time: four elements per lane, the block's two maxima over the wave's lanes.
//   m: nearest float8 e4m3 of (m * (1 / a)) * 256, a the block's largest |m|: steps of 1/16 to 1/8 down to a / 2^14, then of a / 2^17.
//   v: eight bits c, five of exponent and three of fraction; c stands for (the float with the bits c << 20) * 2^96 * a, a the
//      block's largest v, whose code is 248.  Nearest code, ties to even; a v above 0 gets at least code 1: m / sqrt(v) stays
//      bounded where m is still held.
// The largest of a block is held exactly, so a block that shrinks or grows as a whole does so without loss.

constexpr uint32_t kStateBlock = NUQ_STATE_BLOCK;
static_assert(kStateBlock == 256, "a wave holds four elements of a block per lane");
constexpr uint32_t kCodedRows = 4;                              // blocks that a wave takes
constexpr uint32_t kCodedChunk = 4u * kCodedRows * kStateBlock; // elements per workgroup
constexpr uint32_t kCodedTensors = 60;

struct AdamwCodedTable {
    float *w[kCodedTensors], *scales[kCodedTensors];
    uint8_t *m[kCodedTensors], *v[kCodedTensors];
    const void *g[kCodedTensors];
    void *copy[kCodedTensors];
    uint64_t n[kCodedTensors];
    float keep[kCodedTensors];
    uint32_t start[kCodedTensors];
    uint32_t count;
    AdamwNumbers num;
    const float *coefficient;
    uint32_t *flags;
};
static_assert(sizeof(AdamwCodedTable) <= 4096, "a launch's arguments");

typedef uint32_t CodeWord __attribute__((aligned(1), may_alias));

__device__ __forceinline__ uint32_t load_codes(const uint8_t *from, int64_t have)
{
    if (have >= 4)
        return *reinterpret_cast<const CodeWord *>(from);
    uint32_t x = 0;
#pragma unroll
    for (int e = 0; e < 3; ++e)
        x |= e < have ? (uint32_t)from[e] << (8 * e) : 0u;
    return x;
}
__device__ __forceinline__ void store_codes(uint8_t *to, uint32_t x, int64_t have)
{
    if (have >= 4) {
        *reinterpret_cast<CodeWord *>(to) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < have)
                to[e] = (uint8_t)(x >> (8 * e));
    }
}

__device__ __forceinline__ void decode_m(float (&m)[4], uint32_t codes, float a)
{
    const float unit = a * 0x1p-8f;
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    m[0] = lo[0] * unit;
    m[1] = lo[1] * unit;
    m[2] = hi[0] * unit;
    m[3] = hi[1] * unit;
}
__device__ __forceinline__ void decode_v(float (&v)[4], uint32_t codes, float a)
{
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] = __builtin_bit_cast(float, ((codes >> (8 * e)) & 0xFFu) << 20) * 0x1p96f * a;
}
__device__ __forceinline__ uint32_t encode_m(const float (&m)[4], float inv)
{
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(m[0] * inv * 256.0f, m[1] * inv * 256.0f, 0, false);
    x = __builtin_amdgcn_cvt_pk_fp8_f32(m[2] * inv * 256.0f, m[3] * inv * 256.0f, x, true);
    return (uint32_t)x;
}
__device__ __forceinline__ uint32_t encode_v(const float (&v)[4], float inv)
{
    uint32_t x = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, v[e] * inv * 0x1p-96f);
        uint32_t code = (bits + 0x7FFFFu + ((bits >> 20) & 1u)) >> 20;
        code = max(code, v[e] > 0.0f && inv > 0.0f ? 1u : 0u);
        x |= code << (8 * e);
    }
    return x;
}

// One pass: 16 bytes per element with 32-bit gradients.  A block whose new moments are not all finite is left as it is.
template <class G, class C, bool kCopy>
__global__ __launch_bounds__(256) void k_adamw_coded(const AdamwCodedTable P)
{
    const uint32_t t = (uint32_t)__builtin_amdgcn_readfirstlane((int)tensor_of(P.start, P.count, blockIdx.x));
    const uint32_t lane = threadIdx.x % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    const uint64_t n = P.n[t], block0 = (uint64_t)(blockIdx.x - P.start[t]) * (4u * kCodedRows) + wave * kCodedRows;
    const float keep = P.keep[t], c = P.coefficient ? *P.coefficient : 1.0f;
    float *const pw = P.w[t], *const scales = P.scales[t];
    uint8_t *const pm = P.m[t], *const pv = P.v[t];
    const G *const pg = static_cast<const G *>(P.g[t]);
    float w[kCodedRows][4], g[kCodedRows][4], am[kCodedRows], av[kCodedRows];
    uint32_t cm[kCodedRows], cv[kCodedRows];
#pragma unroll
    for (uint32_t r = 0; r < kCodedRows; ++r) {
        const uint64_t i = (block0 + r) * kStateBlock + lane * 4u;
        const int64_t have = (int64_t)n - (int64_t)i;
        const bool some = (block0 + r) * kStateBlock < n;
        am[r] = some ? scales[2u * (block0 + r)] : 0.0f;
        av[r] = some ? scales[2u * (block0 + r) + 1u] : 0.0f;
        cm[r] = load_codes(pm + i, have);
        cv[r] = load_codes(pv + i, have);
        load_some<4>(g[r], pg + i, have);
        load_some<4>(w[r], pw + i, have);
    }
    bool lost = false;
#pragma unroll
    for (uint32_t r = 0; r < kCodedRows; ++r) {
        const uint64_t i = (block0 + r) * kStateBlock + lane * 4u;
        const int64_t have = (int64_t)n - (int64_t)i;
        float m[4], v[4];
        decode_m(m, cm[r], am[r]);
        decode_v(v, cv[r], av[r]);
        uint32_t top_m = 0, top_v = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            adamw_moments(m[e], v[e], g[r][e] * c, P.num);
            top_m = max(top_m, e < have ? __builtin_bit_cast(uint32_t, m[e]) & 0x7FFFFFFFu : 0u);
            top_v = max(top_v, e < have ? __builtin_bit_cast(uint32_t, v[e]) : 0u);
        }
        top_m = wave_max(top_m);
        top_v = wave_max(top_v);
        if (max(top_m, top_v) >= 0x7F800000u) {
            lost = true;
            if constexpr (kCopy)
                store_some<4>(static_cast<C *>(P.copy[t]) + i, w[r], have);
            continue;
        }
        top_m = top_m < 0x00800000u ? 0u : top_m;
        top_v = top_v < 0x00800000u ? 0u : top_v;
        const float a = __builtin_bit_cast(float, top_m), b = __builtin_bit_cast(float, top_v);
        store_codes(pm + i, encode_m(m, top_m ? 1.0f / a : 0.0f), have);
        store_codes(pv + i, encode_v(v, top_v ? 1.0f / b : 0.0f), have);
        if (lane == 0 && have > 0) {
            scales[2u * (block0 + r)] = a;
            scales[2u * (block0 + r) + 1u] = b;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[r][e] = adamw_weight(w[r][e], m[e], v[e], keep, P.num);
        store_some<4>(pw + i, w[r], have);
        if constexpr (kCopy)
            store_some<4>(static_cast<C *>(P.copy[t]) + i, w[r], have);
    }
    if (lost && lane == 0)
        atomicOr(P.flags, NUQ_FLAG_NONFINITE);
}

// The values that the codes of one tensor stand for.
__global__ __launch_bounds__(256) void k_adamw_values(const uint8_t *pm, const uint8_t *pv, const float *scales, float *m,
                                                      float *v, uint64_t n)
{
    const uint64_t i = ((uint64_t)blockIdx.x * 256u + threadIdx.x) * 4u, block = i / kStateBlock;
    const int64_t have = (int64_t)n - (int64_t)i;
    if (have <= 0)
        return;
    float x[4];
    decode_m(x, load_codes(pm + i, have), scales[2u * block]);
    store_some<4>(m + i, x, have);
    decode_v(x, load_codes(pv + i, have), scales[2u * block + 1u]);
    store_some<4>(v + i, x, have);
}

// ---- the norm of all gradients ----
// Sums of squares in fp64 (products of fp32 values are exact there, and no square overflows): a partial per workgroup, then one
// workgroup adds them in a fixed order.

constexpr uint32_t kNormTensors = 128;
constexpr uint32_t kNormChunk = 256u * 4u * 4u;
constexpr uint32_t kNormPartials = NUQ_GRADIENT_NORM_WORKSPACE_BYTES / sizeof(double);

struct NormTable {
    const void *g[kNormTensors];
    uint64_t n[kNormTensors];
    uint32_t start[kNormTensors + 1];       // start[count]: the chunks of all
    uint32_t count;
    double *partial;
};
static_assert(sizeof(NormTable) <= 4096, "a launch's arguments");

// Workgroup p takes the p-th share of the chunks and writes partial[p].
template <class G>
__global__ __launch_bounds__(256) void k_gradient_norm(const NormTable P)
{
    __shared__ double red[4];
    const uint64_t chunks = P.start[P.count];
    const uint32_t first = (uint32_t)(chunks * blockIdx.x / gridDim.x), last = (uint32_t)(chunks * (blockIdx.x + 1u) / gridDim.x);
    uint32_t t = 0;
    for (uint32_t k = 0; k < P.count; k += 64u) {           // (the last of these steps that finds anything holds it)
        const uint32_t left = P.count - k < 64u ? P.count - k : 64u;
        if (P.start[k] <= first)
            t = k + (uint32_t)__builtin_amdgcn_readfirstlane((int)tensor_of(P.start + k, left, first));
    }
    double sum = 0.0;
    for (uint32_t chunk = first; chunk < last; ++chunk) {
        while (chunk >= P.start[t + 1u])
            ++t;
        const G *const pg = static_cast<const G *>(P.g[t]);
        const uint64_t base = (uint64_t)(chunk - P.start[t]) * kNormChunk, n = P.n[t];
        float g[4][4];
#pragma unroll
        for (uint32_t r = 0; r < 4u; ++r) {
            const uint64_t i = base + (r * 256u + threadIdx.x) * 4u;
            load_some<4>(g[r], pg + i, (int64_t)n - (int64_t)i);
        }
#pragma unroll
        for (uint32_t r = 0; r < 4u; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum += (double)g[r][e] * (double)g[r][e];
    }
    sum = workgroup_sum<256>(sum, red);
    if (threadIdx.x == 0)
        P.partial[blockIdx.x] = sum;
}

// out[0] = the norm, out[1] = min(1, max_norm / norm); a norm that is not finite makes both NaN or infinite as it is, and the
// factor NaN: a step behind it changes nothing.
__global__ __launch_bounds__(1024) void k_gradient_norm_finish(const double *partial, uint32_t count, float max_norm, float *out,
                                                               uint32_t *flags)
{
    __shared__ double red[16];
    double sum = 0.0;
    for (uint32_t p = threadIdx.x; p < count; p += 1024u)
        sum += partial[p];
    sum = workgroup_sum<1024>(sum, red);
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum);
        const float rounded = (float)norm;
        const bool fine = rounded < __builtin_inff();
        out[0] = rounded;
        out[1] = !fine ? __builtin_nanf("") : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f;
        if (!fine)
            atomicOr(flags, NUQ_FLAG_NONFINITE);
    }
}

}  // namespace nuq
