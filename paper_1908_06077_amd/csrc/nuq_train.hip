// C ABI of the optimizer and the layer norm (see include/nuq.h): argument checks, the tables of tensors and the launches.  A
// source file of its own, so that it is built beside the other.
#include "../../include/nuq.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <iterator>
#include <type_traits>

#include "nuq_adamw_kernels.hpp"
#include "nuq_layer_norm_kernels.hpp"
#include "nuq_train_host.hpp"

namespace {

using namespace nuq;

// What a step's launches have in common, and what the step's arguments are checked for.
struct AdamwCall {
    uint32_t T, g_type, copy_type;
    const void *const *g;
    void *const *copy;
    const uint64_t *n;
    const float *decay;
    double alpha, beta1, beta2, eps;
    uint64_t t;
    const float *coefficient;

    bool valid(float *const *w) const
    {
        if (g_type > NUQ_F16 || (copy && copy_type != NUQ_BF16 && copy_type != NUQ_F16) || t == 0 || !std::isfinite(alpha) ||
            !std::isfinite(beta1) || !std::isfinite(beta2) || beta1 < 0.0 || !(beta1 < 1.0) || beta2 < 0.0 || !(beta2 < 1.0) ||
            !(eps >= 0x1p-126) || !std::isfinite((float)eps) || (coefficient && off_grid(coefficient, 4)) ||
            (T > 0 && (!w || !g || !n)))
            return false;
        for (uint32_t i = 0; i < T; ++i)
            if (!valid_array(w[i], n[i], 4) || !valid_array(g[i], n[i], width(g_type)) ||
                (copy && !valid_array(copy[i], n[i], 2)) || n[i] > UINT64_MAX / 16u || !std::isfinite(keep(i)))
                return false;
        return std::isfinite((float)(alpha / faded(beta1)));
    }
    double faded(double beta) const { return -std::expm1((double)t * std::log(beta)); }        // 1 - beta^t
    // Whether a step replaces less than a sixteenth of a moment.
    bool creeps(double beta) const { return 16.0 * (1.0 - beta) < faded(beta); }
    AdamwNumbers numbers() const
    {
        // The hardware's reciprocal of a number above 2^126 is 0: near there the denominator is taken 2^-16 times as large, and with
        // it the step.  (The root is at most 2^64, its factor 2^27.)
        const double part = eps > 0x1p120 ? 0x1p-16 : 1.0;
        return {(float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)(alpha / faded(beta1) * part),
                (float)(1.0 / std::sqrt(faded(beta2)) * part), (float)(eps * part)};
    }
    float keep(uint32_t i) const { return decay ? (float)(1.0 - alpha * (double)decay[i]) : 1.0f; }
    const void *g_at(uint32_t i, uint64_t e) const { return static_cast<const char *>(g[i]) + e * width(g_type); }
    void *copy_at(uint32_t i, uint64_t e) const { return copy ? static_cast<char *>(copy[i]) + e * 2u : nullptr; }

    // Whether tensor j's elements follow those of tensor i, whose run is `before` elements long, in the arrays all steps have.
    bool follows(float *const *w, uint32_t i, uint32_t j, uint64_t before) const
    {
        return w[j] == w[i] + before && g[j] == g_at(i, before) && keep(i) == keep(j) &&
               (!copy || copy[j] == static_cast<char *>(copy[i]) + before * 2u);
    }
    // f(gradient type, copy type, whether there is a copy, whether the arrays, `bytes` per element and gradient and copy, are
    // larger than the last-level cache)
    template <class F>
    int with_types(uint32_t bytes, F &&f) const
    {
        uint64_t all = 0;
        for (uint32_t i = 0; i < T; ++i)
            all += n[i];
        const bool once = all > kLastLevelCache / (bytes + width(g_type) + (copy ? 2u : 0u));
        return with_type(g_type, [&](auto gt) {
            const auto with_copy = [&](auto ct, auto has) { return once ? f(gt, ct, has, std::true_type{}) : f(gt, ct, has, std::false_type{}); };
            return !copy                     ? with_copy(Type<__bf16>{}, std::false_type{})
                   : copy_type == NUQ_BF16 ? with_copy(Type<__bf16>{}, std::true_type{})
                                           : with_copy(Type<_Float16>{}, std::true_type{});
        });
    }
};

// Chunks whose norm one workgroup takes in a launch of its own: 4.1 us at 4 of them, 4.5 at 16, 6.3 to 6.4 at 25, 9.4 at 49, where two
// launches take 6.0 to 6.8.
constexpr uint32_t kSmallChunks = 24;

// Walks the tensors of a call, joined where one follows another, and fills tables of at most kMost of them: put(slot, tensor,
// first element, elements, first chunk) for each, launch(entries, chunks) for each table.  Runs are cut so that a launch has at
// most kMostGroups chunks.
template <uint32_t kMost, class Follows, class Put, class Launch>
int for_tables(uint32_t T, const uint64_t *n, uint64_t chunk, Follows &&follows, Put &&put, Launch &&launch)
{
    uint32_t slots = 0;
    uint64_t chunks = 0;
    const auto flush = [&]() -> int {
        const int rc = slots ? launch(slots, (uint32_t)chunks) : (int)NUQ_OK;
        slots = 0;
        chunks = 0;
        return rc;
    };
    for (uint32_t i = 0; i < T;) {
        uint64_t run = n[i];
        uint32_t j = i + 1;
        while (run && j < T && (n[j] == 0 || follows(i, j, run)))
            run += n[j++];
        for (uint64_t at = 0; at < run;) {
            if (slots == kMost || chunks == kMostGroups)
                if (const int rc = flush(); rc != NUQ_OK)
                    return rc;
            const uint64_t take = std::min(run - at, (kMostGroups - chunks) * chunk);
            put(slots++, i, at, take, (uint32_t)chunks);
            chunks += (take + chunk - 1) / chunk;
            at += take;
        }
        i = j;
    }
    return flush();
}

}  // namespace

extern "C" {

int nuq_gradient_norm(uint32_t T, const void *const *g, const uint64_t *n, uint32_t type, float max_norm, void *workspace,
                      uint64_t workspace_bytes, float *out, nuq_stream_t stream)
{
    if (type > NUQ_F16 || !(max_norm > 0.0f) || !workspace || off_grid(workspace, 8) ||
        workspace_bytes < NUQ_GRADIENT_NORM_WORKSPACE_BYTES || !out || off_grid(out, 4) || (T > 0 && (!g || !n)))
        return NUQ_EINVAL;
    uint64_t all = 0;
    for (uint32_t i = 0; i < T; ++i) {
        if (!valid_array(g[i], n[i], width(type)) || n[i] > UINT64_MAX / 16u)
            return NUQ_EINVAL;
        all += n[i];
    }
    const bool once = all > kLastLevelCache / width(type);
    uint32_t *const flags = flags_ptr();
    if (!flags)
        return NUQ_EHIP;
    const uint32_t w = width(type);
    const auto follows = [&](uint32_t i, uint32_t j, uint64_t before) {
        return g[j] == static_cast<const char *>(g[i]) + before * w;
    };
    hipStream_t st = static_cast<hipStream_t>(stream);
    NormTable P;
    double *const partial = static_cast<double *>(workspace);
    // the launches share the partials
    uint32_t launches = 0, only = 0;
    (void)for_tables<kTableTensors>(T, n, kNormChunk, follows, [](auto...) {}, [&](uint32_t, uint32_t chunks) {
        ++launches;
        only = chunks;
        return (int)NUQ_OK;
    });
    const bool small = launches == 1 && only <= kSmallChunks;
    if (launches > kNormPartials)
        return NUQ_EINVAL;
    const uint32_t most = launches ? kNormPartials / launches : 0u;
    uint32_t used = 0;
    const int rc = for_tables<kTableTensors>(
        T, n, kNormChunk, follows,
        [&](uint32_t slot, uint32_t i, uint64_t at, uint64_t take, uint32_t start) {
            P.tensor[slot] = {static_cast<const char *>(g[i]) + at * w, take};
            P.start[slot] = start;
        },
        [&](uint32_t slots, uint32_t chunks) {
            std::fill(P.start + slots, std::end(P.start), ~0u);
            P.chunks = chunks;
            if (small)
                return with_type(type, [&](auto t) {
                    hipLaunchKernelGGL(k_gradient_norm_small<typename decltype(t)::type>, dim3(1), dim3(1024), 0, st, P, max_norm,
                                       out, flags);
                    return check_launch();
                });
            P.partial = partial + used;
            const uint32_t grid = std::min(chunks, most);
            used += grid;
            return with_type(type, [&](auto t) {
                using G = typename decltype(t)::type;
                if (once)
                    hipLaunchKernelGGL((k_gradient_norm<G, true>), dim3(grid), dim3(256), 0, st, P);
                else
                    hipLaunchKernelGGL((k_gradient_norm<G, false>), dim3(grid), dim3(256), 0, st, P);
                return check_launch();
            });
        });
    if (rc != NUQ_OK || small)
        return rc;
    hipLaunchKernelGGL(k_gradient_norm_finish, dim3(1), dim3(1024), 0, st, partial, used, max_norm, out, flags);
    return check_launch();
}

int nuq_adamw_step(uint32_t T, float *const *w, const void *const *g, float *const *m, float *const *v, void *const *copy,
                   const uint64_t *n, const float *decay, uint32_t g_type, uint32_t copy_type, double alpha, double beta1,
                   double beta2, double eps, uint64_t t, const float *coefficient, nuq_stream_t stream)
{
    const AdamwCall C{T, g_type, copy_type, g, copy, n, decay, alpha, beta1, beta2, eps, t, coefficient};
    if (!C.valid(w) || (T > 0 && (!m || !v)))
        return NUQ_EINVAL;
    for (uint32_t i = 0; i < T; ++i)
        if (!valid_array(m[i], n[i], 4) || !valid_array(v[i], n[i], 4))
            return NUQ_EINVAL;
    AdamwTable P;
    P.num = C.numbers();
    P.coefficient = coefficient;
    P.flags = flags_ptr();
    if (!P.flags)
        return NUQ_EHIP;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return for_tables<kTableTensors>(
        T, n, kAdamwChunk,
        [&](uint32_t i, uint32_t j, uint64_t before) {
            return C.follows(w, i, j, before) && m[j] == m[i] + before && v[j] == v[i] + before;
        },
        [&](uint32_t slot, uint32_t i, uint64_t at, uint64_t take, uint32_t start) {
            P.tensor[slot] = {w[i] + at, m[i] + at, v[i] + at, C.g_at(i, at), C.copy_at(i, at), take, C.keep(i)};
            P.start[slot] = start;
        },
        [&](uint32_t slots, uint32_t chunks) {
            std::fill(P.start + slots, std::end(P.start), ~0u);
            return C.with_types(12, [&](auto gt, auto ct, auto has, auto once) {
                hipLaunchKernelGGL((k_adamw<typename decltype(gt)::type, typename decltype(ct)::type, decltype(has)::value,
                                            decltype(once)::value>), dim3(chunks), dim3(256), 0, st, P);
                return check_launch();
            });
        });
}

uint64_t nuq_state_blocks(uint64_t n) { return n / NUQ_STATE_BLOCK + (n % NUQ_STATE_BLOCK != 0); }

int nuq_adamw_step_coded(uint32_t T, float *const *w, const void *const *g, uint8_t *const *m, uint8_t *const *v,
                         float *const *scales, void *const *copy, const uint64_t *n, const float *decay, uint32_t g_type,
                         uint32_t copy_type, double alpha, double beta1, double beta2, double eps, uint64_t t,
                         const float *coefficient, nuq_stream_t stream)
{
    const AdamwCall C{T, g_type, copy_type, g, copy, n, decay, alpha, beta1, beta2, eps, t, coefficient};
    if (!C.valid(w) || (T > 0 && (!m || !v || !scales)))
        return NUQ_EINVAL;
    for (uint32_t i = 0; i < T; ++i)
        if (!valid_array(m[i], n[i], 1) || !valid_array(v[i], n[i], 1) || !valid_array(scales[i], n[i], 4))
            return NUQ_EINVAL;
    AdamwCodedTable P;
    P.num = C.numbers();
    P.t = t;
    P.draw_m = C.creeps(beta1);
    P.draw_v = C.creeps(beta2);
    P.coefficient = coefficient;
    P.flags = flags_ptr();
    if (!P.flags)
        return NUQ_EHIP;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return for_tables<kCodedTensors>(
        T, n, kCodedChunk,
        [&](uint32_t i, uint32_t j, uint64_t before) {
            return before % NUQ_STATE_BLOCK == 0 && C.follows(w, i, j, before) && m[j] == m[i] + before &&
                   v[j] == v[i] + before && scales[j] == scales[i] + 2u * (before / NUQ_STATE_BLOCK);
        },
        [&](uint32_t slot, uint32_t i, uint64_t at, uint64_t take, uint32_t start) {     // (`at`: whole chunks)
            P.tensor[slot] = {w[i] + at, scales[i] + 2u * (at / NUQ_STATE_BLOCK), m[i] + at, v[i] + at, C.g_at(i, at),
                              C.copy_at(i, at), take, C.keep(i)};
            P.start[slot] = start;
        },
        [&](uint32_t slots, uint32_t chunks) {
            std::fill(P.start + slots, std::end(P.start), ~0u);
            return C.with_types(6, [&](auto gt, auto ct, auto has, auto once) {
                hipLaunchKernelGGL((k_adamw_coded<typename decltype(gt)::type, typename decltype(ct)::type, decltype(has)::value,
                                                  decltype(once)::value>), dim3(chunks), dim3(256), 0, st, P);
                return check_launch();
            });
        });
}

int nuq_adamw_state_values(const uint8_t *m_codes, const uint8_t *v_codes, const float *scales, uint64_t n, float *m, float *v,
                           nuq_stream_t stream)
{
    if (n == 0)
        return NUQ_OK;
    if (!m_codes || !v_codes || !valid_array(scales, n, 4) || !valid_array(m, n, 4) || !valid_array(v, n, 4) || n > UINT64_MAX / 16u)
        return NUQ_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool once = n > kLastLevelCache / 10u;
    for (uint64_t at = 0; at < n; at += kMostGroups * 1024u) {
        const uint64_t take = std::min(n - at, kMostGroups * 1024u);
        const dim3 grid((uint32_t)((take + 1023u) / 1024u));
        const float *const a = scales + 2u * (at / NUQ_STATE_BLOCK);
        if (once)
            hipLaunchKernelGGL(k_adamw_values<true>, grid, dim3(256), 0, st, m_codes + at, v_codes + at, a, m + at, v + at, take);
        else
            hipLaunchKernelGGL(k_adamw_values<false>, grid, dim3(256), 0, st, m_codes + at, v_codes + at, a, m + at, v + at, take);
    }
    return check_launch();
}

}  // extern "C"

namespace {

// The team of threads, the elements per thread and the vectors that hold a row of `hidden` elements of type T: f(team, elements,
// vector), or f(0, 0, 0) where nothing does.  Forward and backward pass differ where registers do:
//   513 to 1024 columns in float32: a backward team of 128 (33554 x 1000 with a gradient to add 105 us, 113 with a wave; in 16
//     bits a wave, 3 % faster);
//   1025 to 2048: a forward team of 128 (20971 x 1600 in bfloat16 28.6 us, 32.1 with 256 threads of eight elements; the backward
//     pass gains nothing);
//   8193 to 12288: forward 512 threads of 24 elements (40.8 us on 4096 rows in bfloat16, 44.0 with 768 of sixteen), backward 768
//     of sixteen, whose sums stand in LDS.
// Teams of 192 and 384 threads between were tried: 5 % less at 1300 columns, 10 % more at 2500 and 5000.
template <class T, bool kBackward, class F>
int with_row_shape(uint32_t hidden, F &&f)
{
    using std::integral_constant;
    constexpr int VEC = 16 / (int)sizeof(T);                // a 16-byte access
    if (hidden < VEC)
        return f(integral_constant<int, 4>{}, integral_constant<int, 2>{}, integral_constant<int, 1>{});
#define NUQ_SHAPE(team, elements)                                                                                     \
    if (hidden <= team * elements)                                                                                    \
        return f(integral_constant<int, team>{}, integral_constant<int, elements>{}, integral_constant<int, VEC>{});
    NUQ_SHAPE(4, 8)
    NUQ_SHAPE(16, 8)
    NUQ_SHAPE(16, 16)
    NUQ_SHAPE(32, 16)
    if constexpr (kBackward && VEC == 4) {
        NUQ_SHAPE(128, 8)
    } else {
        NUQ_SHAPE(64, 16)
    }
    if constexpr (kBackward) {
        NUQ_SHAPE(256, 8)
        NUQ_SHAPE(256, 16)
        NUQ_SHAPE(512, 16)
        NUQ_SHAPE(768, 16)
    } else {
        NUQ_SHAPE(128, 16)
        NUQ_SHAPE(256, 16)
        NUQ_SHAPE(512, 16)
        NUQ_SHAPE(512, 24)
    }
    NUQ_SHAPE(1024, 16)
#undef NUQ_SHAPE
    return f(integral_constant<int, 0>{}, integral_constant<int, 0>{}, integral_constant<int, 0>{});
}

bool valid_rows(uint64_t rows, uint32_t hidden, uint32_t type, uint32_t weight_type, const void *weight)
{
    return hidden >= 1 && hidden <= 1u << 30 && rows < 1ull << 31 && type <= NUQ_F16 &&
           (weight_type == type || weight_type == NUQ_F32) && (!weight || !off_grid(weight, width(weight_type)));
}

// Workgroups that write partial sums of the weights' gradients (at most: 1024 of them on 8192 x 1600 take 2 us more than 512, 256
// one), and such rows of workgroups for long rows.
constexpr uint32_t kParts = 512, kLongParts = 64;
static_assert(kParts <= 1024, "nuq_layer_norm_workspace_bytes");

dim3 long_grid(uint64_t rows) { return dim3((uint32_t)std::min<uint64_t>(rows, kMostGroups * 256u / kLongRowWG)); }

}  // namespace

extern "C" {

int nuq_layer_norm_forward(const void *x, uint64_t ldx, const void *residual, uint64_t ldr, const void *weight,
                           const void *bias, uint64_t rows, uint32_t hidden, float eps, uint32_t type, uint32_t weight_type,
                           void *total, uint64_t ldt, void *y, uint64_t ldy, float *mean, float *rstd, nuq_stream_t stream)
{
    if (!valid_rows(rows, hidden, type, weight_type, weight) || (bias && off_grid(bias, width(weight_type))) ||
        !std::isfinite(eps) || eps < 0.0f || !residual != !total || (mean && off_grid(mean, 4)) || (rstd && off_grid(rstd, 4)))
        return NUQ_EINVAL;
    if (rows == 0)
        return NUQ_OK;
    const uint32_t w = width(type);
    if (!valid_array(x, 1, w) || !valid_array(y, 1, w) || (residual && (off_grid(residual, w) || off_grid(total, w))) ||
        (rows > 1 && (ldy < hidden || (total && ldt < hidden))))
        return NUQ_EINVAL;
    // A result larger than the last-level cache takes long enough for workgroups to drift apart: a quarter of the rows for each
    // evens that out (8192 x 12288 in float32 147 -> 142 us; 8192 x 1600 in bfloat16 21.6 -> 23.3 would be slower).
    const bool long_batch = rows * hidden > kLastLevelCache / w;
    const LayerNormForward P{x, residual, weight, bias, total, y, mean, rstd, rows, ldx, ldr, ldt, ldy, hidden, eps};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return with_types(type, weight_type, [&](auto tt, auto wt) {
        using T = typename decltype(tt)::type;
        using W = typename decltype(wt)::type;
        return with_row_shape<T, false>(hidden, [&](auto team, auto elements, auto vec) {
            constexpr int TEAM = decltype(team)::value, E = decltype(elements)::value, VEC = decltype(vec)::value;
            const auto run = [&](auto stream_c) {
                constexpr bool kStream = decltype(stream_c)::value;
                if constexpr (TEAM == 0) {
                    hipLaunchKernelGGL((k_layer_norm_forward_long<T, W, kStream>), long_grid(rows), dim3(kLongRowWG), 0, st, P);
                } else {
                    constexpr uint32_t WG = kForwardWG<TEAM>, TEAMS = WG / TEAM;
                    const uint32_t most = resident_workgroups<k_layer_norm_forward<T, W, TEAM, E, VEC, kStream>>(WG);
                    if (!most)
                        return (int)NUQ_EHIP;
                    const uint32_t grid = (uint32_t)std::min<uint64_t>((rows + TEAMS - 1) / TEAMS, long_batch ? 4u * most : most);
                    hipLaunchKernelGGL((k_layer_norm_forward<T, W, TEAM, E, VEC, kStream>), dim3(grid), dim3(WG), 0, st, P);
                }
                return check_launch();
            };
            return residual ? run(std::true_type{}) : run(std::false_type{});
        });
    });
}

uint64_t nuq_layer_norm_workspace_bytes(uint64_t rows, uint32_t hidden)
{
    return 8ull * hidden * std::min<uint64_t>(rows, 1024u);
}

int nuq_layer_norm_backward(const void *dy, uint64_t ldg, const void *x, uint64_t ldx, const void *weight, const float *mean,
                            const float *rstd, const void *add, uint64_t lda, uint64_t rows, uint32_t hidden, uint32_t type,
                            uint32_t weight_type, void *dx, uint64_t ldd, void *dweight, void *dbias, void *workspace,
                            uint64_t workspace_bytes, nuq_stream_t stream)
{
    const bool sums = dweight || dbias;
    if (!valid_rows(rows, hidden, type, weight_type, weight) || (dweight && off_grid(dweight, width(weight_type))) ||
        (dbias && off_grid(dbias, width(weight_type))))
        return NUQ_EINVAL;
    const uint32_t w = width(type);
    if (rows > 0 && (!valid_array(dy, 1, w) || !valid_array(x, 1, w) || !valid_array(dx, 1, w) || !valid_array(mean, 1, 4) ||
                     !valid_array(rstd, 1, 4) || (add && off_grid(add, w)) || (rows > 1 && ldd < hidden) ||
                     (sums && (!workspace || off_grid(workspace, 16)))))
        return NUQ_EINVAL;
    if (rows > 0 && sums && workspace_bytes < nuq_layer_norm_workspace_bytes(rows, hidden))
        return NUQ_ECAPACITY;
    const LayerNormBackward P{dy, x, weight, add, mean, rstd, dx, static_cast<float *>(workspace), rows, ldg, ldx, lda, ldd, hidden};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return with_types(type, weight_type, [&](auto tt, auto wt) {
        using T = typename decltype(tt)::type;
        using W = typename decltype(wt)::type;
        uint32_t parts = 0;
        const int rc = rows == 0 ? (int)NUQ_OK : with_row_shape<T, true>(hidden, [&](auto team, auto elements, auto vec) {
            constexpr int TEAM = decltype(team)::value, E = decltype(elements)::value, VEC = decltype(vec)::value;
            if constexpr (TEAM == 0) {
                constexpr uint32_t VEC_T = 16u / sizeof(T);
                parts = (uint32_t)std::min<uint64_t>(rows, kLongParts);
                if (sums)
                    hipLaunchKernelGGL((k_layer_norm_columns<T>), dim3((hidden + 256u * VEC_T - 1u) / (256u * VEC_T), parts), dim3(256), 0, st, P);
                hipLaunchKernelGGL((k_layer_norm_backward_long<T, W>), long_grid(rows), dim3(kLongRowWG), 0, st, P);
                return check_launch();
            } else {
                constexpr uint32_t WG = kBackwardWG<TEAM, E>, TEAMS = WG / TEAM;
                const auto run = [&](auto sums_c) {
                    constexpr bool kSums = decltype(sums_c)::value;
                    const uint32_t most = resident_workgroups<k_layer_norm_backward<T, W, TEAM, E, VEC, kSums>>(WG);
                    if (!most)
                        return (int)NUQ_EHIP;
                    parts = (uint32_t)std::min<uint64_t>((rows + TEAMS - 1) / TEAMS, kSums ? std::min(most, kParts) : most);
                    hipLaunchKernelGGL((k_layer_norm_backward<T, W, TEAM, E, VEC, kSums>), dim3(parts), dim3(WG), 0, st, P);
                    return check_launch();
                };
                return sums ? run(std::true_type{}) : run(std::false_type{});
            }
        });
        if (rc != NUQ_OK || !sums)
            return rc;
        const uint32_t groups = (uint32_t)std::min<uint64_t>((hidden + 15u) / 16u, kMostGroups * 256u / 1024u / 2u);
        hipLaunchKernelGGL((k_layer_norm_finish<W>), dim3(groups, 2), dim3(1024), 0, st, P.partial, parts, hidden,
                           static_cast<W *>(dweight), static_cast<W *>(dbias));
        return check_launch();
    });
}

}  // extern "C"
