// AdamW over many tensors in one launch, with states in 32 bits or in 8, and the norm of all gradients with the factor that
// clips them.
//
//   g = c * gradient;  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   w <- w (1 - alpha lambda) - alpha / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// m and v are evaluated in fp32, every product and every sum rounded (the 8-bit codes have to come out the same wherever they
// are computed); w takes a hardware square root and reciprocal (1 unit of the last place each) on a term that is a thousandth
// of the weight, and fused multiply-adds.
//
// All of it is bound by HBM: each array is read once and written once (counted: 1.00 times those bytes).  Arrays larger than the
// last-level cache are read and written with non-temporal accesses, both: loads or stores alone change nothing, both take
// 25.6 M elements from 163 to 130 us behind their norm.  Many short workgroups, not persistent ones: a thread's four elements
// are 64 bytes of loads in flight, and 32 waves per CU of them cover the latency; two or four vectors per thread were 2 %
// slower.  Which tensor a workgroup works on comes from the launch's arguments in two dependent loads, where each tensor
// begins (an entry per lane, one ballot), then its pointers: 3.6 us for a launch on 65 537 elements, 4.4 with one array per
// kind of pointer and a count to wait for first.
#pragma once

#include "nuq_train_device.hpp"

namespace nuq {

struct AdamwNumbers {
    float b1, c1, b2, c2;   // beta1, 1 - beta1, beta2, 1 - beta2
    float step;             // alpha / (1 - beta1^t)
    float root;             // 1 / sqrt(1 - beta2^t)
    float eps;              // (all three 2^-16 times as large where eps is huge)
};

__device__ __forceinline__ void adamw_moments(float &m, float &v, float g, const AdamwNumbers &N)
{
    m = m * N.b1 + g * N.c1;              // (the file is compiled without contraction)
    v = v * N.b2 + (g * g) * N.c2;
}

// The hardware's square root reads a subnormal number as 0: small ones are taken 2^32 times as large.
__device__ __forceinline__ float square_root(float v)
{
    const bool small = v < 0x1p-96f;
    return __builtin_amdgcn_sqrtf(small ? v * 0x1p32f : v) * (small ? 0x1p-16f : 1.0f);
}

__device__ __forceinline__ float adamw_weight(float w, float m, float v, float keep, const AdamwNumbers &N)
{
    const float u = m * __builtin_amdgcn_rcpf(__builtin_fmaf(square_root(v), N.root, N.eps));
    return __builtin_fmaf(-N.step, u, w * keep);
}

constexpr uint32_t kAdamwChunk = 256u * 4u;     // elements per workgroup: four per thread

// What a launch's arguments hold for one tensor, side by side: a wave fetches it at once.
struct AdamwTensor {
    float *w, *m, *v;
    const void *g;
    void *copy;
    uint64_t n;
    float keep;                             // 1 - alpha * lambda
};
struct AdamwTable {
    uint32_t start[kTableTensors];
    AdamwTensor tensor[kTableTensors];
    AdamwNumbers num;
    const float *coefficient;               // c, or none
    uint32_t *flags;
};
static_assert(sizeof(AdamwTable) <= 4096, "a launch's arguments");

// One pass: 28 bytes per element with 32-bit gradients (25.6 M elements in 110 us: 6.5 TB/s; 1.56 G with gradients and a copy in
// bfloat16 in 6.9 to 7.6 ms: 5.8 to 6.3).  An element whose new moments are not finite is left as it is.
// kOnce: the call's arrays are larger than the last-level cache.  kWhole: the workgroup's elements are all there.
template <class G, class C, bool kCopy, bool kOnce, bool kWhole>
__device__ __forceinline__ void adamw_chunk(const AdamwTable &P, const AdamwTensor &X, uint64_t base)
{
    const uint64_t i = base + threadIdx.x * 4u;
    const int64_t have = (int64_t)X.n - (int64_t)i;
    float w[4], m[4], v[4], g[4];
    load_some<4, kWhole, kOnce>(g, static_cast<const G *>(X.g) + i, have);
    load_some<4, kWhole, kOnce>(m, X.m + i, have);
    load_some<4, kWhole, kOnce>(v, X.v + i, have);
    load_some<4, kWhole, kOnce>(w, X.w + i, have);
    const float keep = X.keep, c = P.coefficient ? *P.coefficient : 1.0f;
    float m1[4], v1[4];
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        m1[e] = m[e];
        v1[e] = v[e];
        adamw_moments(m1[e], v1[e], g[e] * c, P.num);
        top = max(top, max(__builtin_bit_cast(uint32_t, m1[e]) & 0x7FFFFFFFu, __builtin_bit_cast(uint32_t, v1[e])));
    }
    if (__any(top >= 0x7F800000u)) {                         // (infinities and NaN; what has no element here is zeros)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (max(__builtin_bit_cast(uint32_t, m1[e]) & 0x7FFFFFFFu, __builtin_bit_cast(uint32_t, v1[e])) < 0x7F800000u) {
                m[e] = m1[e];
                v[e] = v1[e];
                w[e] = adamw_weight(w[e], m1[e], v1[e], keep, P.num);
            }
        if (threadIdx.x % 64u == 0)
            atomicOr(P.flags, NUQ_FLAG_NONFINITE);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m[e] = m1[e];
            v[e] = v1[e];
            w[e] = adamw_weight(w[e], m1[e], v1[e], keep, P.num);
        }
    }
    store_some<4, kWhole, kOnce>(X.m + i, m, have);
    store_some<4, kWhole, kOnce>(X.v + i, v, have);
    store_some<4, kWhole, kOnce>(X.w + i, w, have);
    if constexpr (kCopy)
        store_some<4, kWhole, kOnce>(static_cast<C *>(X.copy) + i, w, have);
}

template <class G, class C, bool kCopy, bool kOnce>
__global__ __launch_bounds__(256) void k_adamw(const AdamwTable P)
{
    const uint32_t t = tensor_of(P.start, blockIdx.x);
    const AdamwTensor &X = P.tensor[t];
    const uint64_t base = (uint64_t)(blockIdx.x - P.start[t]) * kAdamwChunk;
    if (base + kAdamwChunk <= X.n)
        adamw_chunk<G, C, kCopy, kOnce, true>(P, X, base);
    else
        adamw_chunk<G, C, kCopy, kOnce, false>(P, X, base);
}

// ---- states in 8 bits ----
// Blocks of 256 elements, one per wave at a time: four elements per lane, the block's two maxima over the wave's lanes.
//   m: float8 e4m3 of (m * (1 / a)) * 256, a the block's largest |m|: steps of 1/16 to 1/8 down to a / 2^14, then of a / 2^17.
//   v: eight bits c, five of exponent and three of fraction; c stands for (the float with the bits c << 20) * 2^96 * a, a the
//      block's largest v, whose code is 248.  A v above 0 gets at least code 1: m / sqrt(v) stays bounded where m is still held.
// The largest of a block is held exactly, so a block that shrinks or grows as a whole does so without loss.
//
// Rounding.  A step replaces the share (1 - beta) / (1 - beta^t) of a moment.  From 1/16 on, which no half step of a code exceeds,
// the nearest code is taken (ties to even).  Below that the nearest code could be the old one for good, so the code is drawn: the upper
// or the lower one, so that the mean is kept.  With beta2 = 0.999 and gradients of one size, sqrt of v as held over sqrt of v in fp32
// has 1 % and 99 % points of 0.76 and 1.28 (0.75 and 1.51 nearest), and after one gradient in sixteen grew fourfold the others come
// back to a median of 0.99 (2.9 nearest).

constexpr uint32_t kStateBlock = NUQ_STATE_BLOCK;
static_assert(kStateBlock == 256, "a wave holds four elements of a block per lane");
constexpr uint32_t kCodedChunk = 4u * kStateBlock;              // elements per workgroup: a block per wave
constexpr uint32_t kCodedTensors = 58;

struct AdamwCodedTensor {
    float *w, *scales;
    uint8_t *m, *v;
    const void *g;
    void *copy;
    uint64_t n;
    float keep;
};
struct AdamwCodedTable {
    uint32_t start[kCodedTensors];
    AdamwCodedTensor tensor[kCodedTensors];
    AdamwNumbers num;
    const float *coefficient;
    uint32_t *flags;
    uint64_t t;
    uint32_t draw_m, draw_v;                // whether codes of m, of v are drawn
};
static_assert(sizeof(AdamwCodedTable) <= 4096, "a launch's arguments");

typedef uint32_t CodeWord __attribute__((aligned(1), may_alias));

template <bool kWhole, bool kOnce>
__device__ __forceinline__ uint32_t load_codes(const uint8_t *from, int64_t have)
{
    if (kWhole || have >= 4) {
        if constexpr (kOnce)
            return __builtin_nontemporal_load(reinterpret_cast<const CodeWord *>(from));
        else
            return *reinterpret_cast<const CodeWord *>(from);
    }
    uint32_t x = 0;
#pragma unroll
    for (int e = 0; e < 3; ++e)
        x |= e < have ? (uint32_t)from[e] << (8 * e) : 0u;
    return x;
}
template <bool kWhole, bool kOnce>
__device__ __forceinline__ void store_codes(uint8_t *to, uint32_t x, int64_t have)
{
    if (kWhole || have >= 4) {
        if constexpr (kOnce)
            __builtin_nontemporal_store(x, reinterpret_cast<CodeWord *>(to));
        else
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
// kDraw: `draw` is added below the code's bits instead of half a step.  least: 1, or 0 in a block of zeros.
template <bool kDraw>
__device__ __forceinline__ uint32_t encode_v(const float (&v)[4], float inv, uint32_t least, const uint32_t (&draw)[4])
{
    uint32_t x = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, v[e] * inv * 0x1p-96f);
        uint32_t code = (bits + (kDraw ? draw[e] : 0x7FFFFu + ((bits >> 20) & 1u))) >> 20;
        code = max(code, min(__builtin_bit_cast(uint32_t, v[e]), least));
        x |= code << (8 * e);
    }
    return x;
}
// The same for m: e4m3 without its sign is the float with the bits c << 20, times 2^120.
__device__ __forceinline__ uint32_t encode_m_drawn(const float (&m)[4], float inv, const uint32_t (&draw)[4])
{
    uint32_t x = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, m[e] * inv * 0x1p-112f);
        x |= (((bits & 0x7FFFFFFFu) + draw[e]) >> 20 | (bits >> 24 & 0x80u)) << (8 * e);
    }
    return x;
}

// Draws for a lane's four codes of v and of m: multiples of 16, and 8, below 2^20, so that what is within seven units of the last
// place of a code's value gets that code (a code that only fades with its scale comes back with the error of five roundings).  They
// come from the step, the block's new scales and the element's place in its block: equal inputs give equal bits, wherever the tensor
// stands and whatever it is joined with.  The counter hash of the quantizer.
__device__ __forceinline__ void state_draws(uint32_t (&for_v)[4], uint32_t (&for_m)[4], uint64_t t, uint32_t top_m, uint32_t top_v,
                                            uint32_t lane)
{
    uint64_t z = ((uint64_t)top_m << 32 | top_v) + t * 0x9E3779B97F4A7C15ull;
    z = (z ^ z >> 30) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ z >> 27) * 0x94D049BB133111EBull;
    z ^= z >> 31;
    const uint32_t first = ((uint32_t)z + lane * 4u) * 0x9E3779B1u;
#pragma unroll
    for (uint32_t e = 0; e < 4u; ++e) {
        uint32_t x = first + e * 0x9E3779B1u;
        x = (x ^ x >> 15 ^ (uint32_t)(z >> 32)) * 0x85EBCA6Bu;
        x ^= x >> 16;
        uint32_t y = x * 0x9E3779B1u;
        y ^= y >> 15;
        for_v[e] = (x >> 12 & 0xFFFF0u) | 8u;
        for_m[e] = (y >> 12 & 0xFFFF0u) | 8u;
    }
}

// One pass: 16 bytes per element with 32-bit gradients (1.56 G with gradients and a copy in bfloat16 in 3.9 ms: 6.3 TB/s; 11.7 M,
// 187 MB, in 37 us: 5.0, of which the start and the last workgroups are some 7).  53 vector instructions per element keep the
// SIMDs busy for less than half of that, 58 with drawn codes of v, 69 of both: 400 M elements take 1030 to 1043 us with them, 1026 to
// 1033 without.  A block per wave: four were 4 % slower on 11.7 M elements.  A block whose new moments are not all finite is left as
// it is.
// kOnce as above; kWhole: the wave's block is all there.
template <class G, class C, bool kCopy, bool kOnce, bool kWhole>
__device__ __forceinline__ void adamw_block(const AdamwCodedTable &P, const AdamwCodedTensor &X, uint64_t block)
{
    const uint32_t lane = threadIdx.x % 64u;
    const uint64_t i = block * kStateBlock + lane * 4u;
    const int64_t have = (int64_t)X.n - (int64_t)i;
    float *const scales = X.scales + 2u * block;
    float w[4], g[4], m[4], v[4];
    const uint32_t codes_m = load_codes<kWhole, kOnce>(X.m + i, have), codes_v = load_codes<kWhole, kOnce>(X.v + i, have);
    const float old_a = scales[0], old_b = scales[1];
    load_some<4, kWhole, kOnce>(g, static_cast<const G *>(X.g) + i, have);
    load_some<4, kWhole, kOnce>(w, X.w + i, have);
    const float keep = X.keep, c = P.coefficient ? *P.coefficient : 1.0f;
    decode_m(m, codes_m, old_a);
    decode_v(v, codes_v, old_b);
    uint32_t top_m = 0, top_v = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        adamw_moments(m[e], v[e], g[e] * c, P.num);
        top_m = max(top_m, kWhole || e < have ? __builtin_bit_cast(uint32_t, m[e]) & 0x7FFFFFFFu : 0u);
        top_v = max(top_v, kWhole || e < have ? __builtin_bit_cast(uint32_t, v[e]) : 0u);
    }
    top_m = wave_max(top_m);
    top_v = wave_max(top_v);
    if (max(top_m, top_v) < 0x7F800000u) {
        top_m = top_m < 0x00800000u ? 0u : top_m;
        top_v = top_v < 0x00800000u ? 0u : top_v;
        const float a = __builtin_bit_cast(float, top_m), b = __builtin_bit_cast(float, top_v);
        const float inv_a = top_m ? 1.0f / a : 0.0f, inv_b = top_v ? 1.0f / b : 0.0f;
        const uint32_t least = top_v ? 1u : 0u;
        uint32_t new_m, new_v;
        if (P.draw_m | P.draw_v) {
            uint32_t for_v[4], for_m[4];
            state_draws(for_v, for_m, P.t, top_m, top_v, lane);
            new_m = P.draw_m ? encode_m_drawn(m, inv_a, for_m) : encode_m(m, inv_a);
            new_v = P.draw_v ? encode_v<true>(v, inv_b, least, for_v) : encode_v<false>(v, inv_b, least, for_v);
        } else {
            const uint32_t none[4] = {};
            new_m = encode_m(m, inv_a);
            new_v = encode_v<false>(v, inv_b, least, none);
        }
        store_codes<kWhole, kOnce>(X.m + i, new_m, have);
        store_codes<kWhole, kOnce>(X.v + i, new_v, have);
        if (lane == 0) {
            scales[0] = a;
            scales[1] = b;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = adamw_weight(w[e], m[e], v[e], keep, P.num);
        store_some<4, kWhole, kOnce>(X.w + i, w, have);
    } else if (lane == 0) {
        atomicOr(P.flags, NUQ_FLAG_NONFINITE);
    }
    if constexpr (kCopy)
        store_some<4, kWhole, kOnce>(static_cast<C *>(X.copy) + i, w, have);
}

template <class G, class C, bool kCopy, bool kOnce>
__global__ __launch_bounds__(256) void k_adamw_coded(const AdamwCodedTable P)
{
    const uint32_t t = tensor_of(P.start, blockIdx.x);
    const AdamwCodedTensor &X = P.tensor[t];
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    const uint64_t block = (uint64_t)(blockIdx.x - P.start[t]) * 4u + wave, n = X.n;
    if ((block + 1u) * kStateBlock <= n)
        adamw_block<G, C, kCopy, kOnce, true>(P, X, block);
    else if (block * kStateBlock < n)
        adamw_block<G, C, kCopy, kOnce, false>(P, X, block);
}

// The values that the codes of one tensor stand for: 10 bytes per element, 6.3 TB/s.
template <bool kOnce>
__global__ __launch_bounds__(256) void k_adamw_values(const uint8_t *pm, const uint8_t *pv, const float *scales, float *m,
                                                      float *v, uint64_t n)
{
    const uint64_t i = ((uint64_t)blockIdx.x * 256u + threadIdx.x) * 4u, block = i / kStateBlock;
    const int64_t have = (int64_t)n - (int64_t)i;
    if (have <= 0)
        return;
    const uint32_t codes_m = load_codes<false, kOnce>(pm + i, have), codes_v = load_codes<false, kOnce>(pv + i, have);
    float x[4], y[4];
    decode_m(x, codes_m, scales[2u * block]);
    decode_v(y, codes_v, scales[2u * block + 1u]);
    store_some<4, false, kOnce>(m + i, x, have);
    store_some<4, false, kOnce>(v + i, y, have);
}

// ---- the norm of all gradients ----
// Sums of squares in fp64 (products of fp32 values are exact there, and no square overflows): a partial per workgroup, then one
// workgroup adds them in a fixed order (a second launch of 4 us: a count of finished workgroups would have to be zero before
// the first call, and the workspace is the caller's).  Bound by HBM: 6.2 GB in 0.90 to 0.93 ms, 6.7 to 6.9 TB/s with non-temporal
// loads, 6.0 without; 102 MB in 18 us.

constexpr uint32_t kNormChunk = 4096u;
constexpr uint32_t kNormPartials = NUQ_GRADIENT_NORM_WORKSPACE_BYTES / sizeof(double);

struct NormTensor {
    const void *g;
    uint64_t n;
};
struct NormTable {
    uint32_t start[kTableTensors];
    NormTensor tensor[kTableTensors];
    uint32_t chunks;                        // of all
    double *partial;
};

template <class G, int WG, bool kOnce, bool kWhole>
__device__ __forceinline__ double square_sum(const G *pg, uint64_t base, uint64_t n)
{
    constexpr int VEC = 16 / sizeof(G), ROWS = (int)kNormChunk / (WG * VEC);
    float g[ROWS][VEC];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint64_t i = base + (uint64_t)(r * WG + (int)threadIdx.x) * VEC;
        load_some<VEC, kWhole, kOnce>(g[r], pg + i, (int64_t)n - (int64_t)i);
    }
    double sum = 0.0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            sum = __builtin_fma((double)g[r][e], (double)g[r][e], sum);
    return sum;
}

// Workgroup p takes the p-th share of the chunks and writes partial[p].  kOnce: the gradients are larger than the last-level
// cache; smaller ones are left there for the step that follows.
template <class G, bool kOnce>
__global__ __launch_bounds__(256) void k_gradient_norm(const NormTable P)
{
    __shared__ double red[4];
    const uint64_t chunks = P.chunks;
    const uint32_t first = (uint32_t)(chunks * blockIdx.x / gridDim.x), last = (uint32_t)(chunks * (blockIdx.x + 1u) / gridDim.x);
    double sum = 0.0;
    for (uint32_t chunk = first; chunk < last; ++chunk) {
        const uint32_t t = tensor_of(P.start, chunk);
        const G *const pg = static_cast<const G *>(P.tensor[t].g);
        const uint64_t base = (uint64_t)(chunk - P.start[t]) * kNormChunk, n = P.tensor[t].n;
        sum += base + kNormChunk <= n ? square_sum<G, 256, kOnce, true>(pg, base, n) : square_sum<G, 256, kOnce, false>(pg, base, n);
    }
    sum = workgroup_sum<256>(sum, red);
    if (threadIdx.x == 0)
        P.partial[blockIdx.x] = sum;
}

// out[0] = the norm, out[1] = min(1, max_norm / norm); NaN where the norm is not finite: a step behind it changes nothing.
__device__ __forceinline__ void norm_and_factor(double sum, float max_norm, float *out, uint32_t *flags)
{
    const double norm = sqrt(sum);
    const float rounded = (float)norm;
    const bool fine = rounded < __builtin_inff();
    out[0] = rounded;
    out[1] = !fine ? __builtin_nanf("") : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f;
    if (!fine)
        atomicOr(flags, NUQ_FLAG_NONFINITE);
}

__global__ __launch_bounds__(1024) void k_gradient_norm_finish(const double *partial, uint32_t count, float max_norm, float *out,
                                                               uint32_t *flags)
{
    __shared__ double red[16];
    double x[kNormPartials / 1024u];
#pragma unroll
    for (uint32_t k = 0; k < kNormPartials / 1024u; ++k)     // all loads at once
        x[k] = threadIdx.x + k * 1024u < count ? partial[threadIdx.x + k * 1024u] : 0.0;
    double sum = 0.0;
#pragma unroll
    for (uint32_t k = 0; k < kNormPartials / 1024u; ++k)
        sum += x[k];
    sum = workgroup_sum<1024>(sum, red);
    if (threadIdx.x == 0)
        norm_and_factor(sum, max_norm, out, flags);
}

// All of it in one workgroup, a quarter of a chunk per wave and two of them at a time: 4.1 us at 16 K elements, 4.5 at 64 K, bound by
// the latency of two loads.  A lane holds the table's entry of one tensor: what a chunk needs comes from there, without another wait
// for memory.  Three or six quarters at a time measured 0.1 and 0.2 us more at 64 K.
template <class G>
__global__ __launch_bounds__(1024) void k_gradient_norm_small(const NormTable P, float max_norm, float *out, uint32_t *flags)
{
    constexpr uint32_t kAtOnce = 2, kWaves = 16, kPart = kNormChunk / 4u;
    __shared__ double red[16];
    const uint32_t lane = threadIdx.x % 64u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64u));
    const uint32_t begin = P.start[lane], parts = P.chunks * 4u;
    const uint64_t where = reinterpret_cast<uint64_t>(P.tensor[lane].g), size = P.tensor[lane].n;
    const auto of = [](uint32_t x, uint32_t t) { return (uint32_t)__builtin_amdgcn_readlane((int)x, (int)t); };
    const auto of64 = [&](uint64_t x, uint32_t t) { return (uint64_t)of((uint32_t)(x >> 32), t) << 32 | of((uint32_t)x, t); };
    double sum = 0.0;
    for (uint32_t first = wave; first < parts; first += kAtOnce * kWaves) {
        float g[kAtOnce][4][4] = {};
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) {
            const uint32_t part = first + k * kWaves, chunk = part / 4u;
            if (part < parts) {
                const uint32_t t = (uint32_t)__popcll(__ballot(begin <= chunk)) - 1u;
                const uint64_t at = (uint64_t)(chunk - of(begin, t)) * kNormChunk + part % 4u * kPart;
                const G *const pg = reinterpret_cast<const G *>(of64(where, t)) + at;
                const int64_t left = (int64_t)of64(size, t) - (int64_t)at;
                if (left >= (int64_t)kPart) {
#pragma unroll
                    for (uint32_t r = 0; r < 4u; ++r)
                        load_as_float<4>(g[k][r], pg + (r * 64u + lane) * 4u);
                } else {
#pragma unroll
                    for (uint32_t r = 0; r < 4u; ++r)
                        load_some<4>(g[k][r], pg + (r * 64u + lane) * 4u, left - (int64_t)((r * 64u + lane) * 4u));
                }
            }
        }
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k)
            if (first + k * kWaves < parts)
#pragma unroll
                for (uint32_t r = 0; r < 4u; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        sum = __builtin_fma((double)g[k][r][e], (double)g[k][r][e], sum);
    }
    sum = workgroup_sum<1024>(sum, red);
    if (threadIdx.x == 0)
        norm_and_factor(sum, max_norm, out, flags);
}

}  // namespace nuq
