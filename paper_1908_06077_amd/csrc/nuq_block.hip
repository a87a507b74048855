// C ABI of dropout and of the norms around a block's residual sum (see include/nuq.h): argument checks and launches.  A source file
// of its own, so that it is built beside the others.
#include "../../include/nuq.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "nuq_dropout_kernels.hpp"
#include "nuq_residual_norm_kernels.hpp"
#include "nuq_train_host.hpp"

namespace {

using namespace nuq;

constexpr uint64_t kMostRows = 1ull << 31;

// False where p is no probability or step is no place for its number.
bool draws_of(double p, uint64_t seed, const int64_t *step, Draws &to)
{
    if (!(p >= 0.0 && p <= 1.0) || off_grid(step, 8))
        return false;
    const uint32_t threshold = (uint32_t)std::floor(p * 0x1p24 + 0.5);
    to = {seed, step, threshold, threshold < 1u << 24 ? (float)(0x1p24 / (0x1p24 - threshold)) : 0.0f};
    return true;
}

enum class SeamPass { kFew, kMany, kBackward };

// The team of threads, the elements per thread and the vectors that hold a row of `hidden` elements of type T.  Every sum over a row costs
// a wave some twenty instructions and a team of several waves a barrier, so teams are small where registers allow it: forward with many
// rows a wave has up to 2048 columns; backward, beside four sums per column, sixteen elements per thread (eight in fp32).  A few rows
// take eight and larger teams, for their latency.
template <class T, SeamPass kPass, class F>
int with_seam_shape(uint32_t hidden, F &&f)
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
    NUQ_SHAPE(64, 8)
    if constexpr (kPass == SeamPass::kMany) {
        if constexpr (VEC == 8) {
            NUQ_SHAPE(64, 16)
            NUQ_SHAPE(128, 16)
        } else {
            NUQ_SHAPE(128, 8)
            NUQ_SHAPE(256, 8)
        }
        return f(integral_constant<int, 0>{}, integral_constant<int, 0>{}, integral_constant<int, 0>{});
    } else {
        NUQ_SHAPE(128, 8)
        NUQ_SHAPE(256, 8)
        NUQ_SHAPE(512, 8)
        if constexpr (kPass == SeamPass::kBackward) {
            NUQ_SHAPE(512, 16)
        } else {
            NUQ_SHAPE(1024, 8)
        }
        return f(integral_constant<int, 1024>{}, integral_constant<int, 16>{}, integral_constant<int, VEC>{});
    }
#undef NUQ_SHAPE
}
constexpr uint32_t kSumsInRegisters = 8192;                  // columns; wider rows have their sums taken by a launch of its own

// Forward, from so many elements on teams take several rows each, and their vectors of weights go into the LDS, where four of so many
// columns leave a CU several workgroups.
constexpr uint64_t kManyElements = 1u << 22;
constexpr uint32_t kManyColumns = 2048;

// Workgroups that write partial sums of the weights' gradients, and such rows of workgroups for wide rows.
constexpr uint32_t kSeamParts = 512, kWideParts = 64;
static_assert(kSeamParts <= 1024, "nuq_residual_norm_workspace_bytes");

bool valid_seam(uint64_t rows, uint32_t hidden, uint32_t type, uint32_t weight_type, uint32_t inner, uint32_t outer, float scale,
                float residual_scale, std::initializer_list<const void *> vectors)
{
    if (hidden < 1 || hidden > NUQ_RESIDUAL_NORM_MAX_HIDDEN || rows >= kMostRows || type > NUQ_F16 ||
        (weight_type != type && weight_type != NUQ_F32) || inner > NUQ_RMS_NORM || outer > NUQ_RMS_NORM ||
        (inner == NUQ_NO_NORM && outer == NUQ_NO_NORM) || !std::isfinite(scale) || !std::isfinite(residual_scale))
        return false;
    for (const void *v : vectors)
        if (off_grid(v, width(weight_type)))
            return false;
    return true;
}

}  // namespace

extern "C" {

int nuq_dropout(const void *x, uint64_t ldx, const void *residual, uint64_t ldr, uint64_t rows, uint32_t hidden, uint32_t type,
                double p, uint64_t seed, const int64_t *step, void *y, uint64_t ldy, nuq_stream_t stream)
{
    Dropout P{x, residual, y, {}, rows, ldx, ldr, ldy, hidden};
    if (hidden >= 1u << 31 || rows >= kMostRows || type > NUQ_F16 || !draws_of(p, seed, step, P.draws))
        return NUQ_EINVAL;
    if (rows == 0 || hidden == 0)
        return NUQ_OK;
    const uint32_t w = width(type);
    if (!valid_array(x, 1, w) || !valid_array(y, 1, w) || off_grid(residual, w) ||
        (rows > 1 && (ldy < hidden || other_stride(y, ldy, x, ldx) || other_stride(y, ldy, residual, ldr))))
        return NUQ_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return with_type(type, [&](auto t) {
        using T = typename decltype(t)::type;
        const uint64_t vectors = (hidden + 16u / w - 1u) / (16u / w) * rows;
        const dim3 grid((uint32_t)std::min<uint64_t>((vectors + 255u) / 256u, 256u * 32u));
        const auto run = [&](auto residual_c, auto once_c) {
            hipLaunchKernelGGL((k_dropout<T, decltype(residual_c)::value, decltype(once_c)::value>), grid, dim3(256), 0, st, P);
            return check_launch();
        };
        const bool once = rows * hidden > kLastLevelCache / (w * (residual ? 3u : 2u));
        const auto with_residual = [&](auto once_c) { return residual ? run(std::true_type{}, once_c) : run(std::false_type{}, once_c); };
        return once ? with_residual(std::true_type{}) : with_residual(std::false_type{});
    });
}

int nuq_residual_norm_forward(const void *x, uint64_t ldx, const void *residual, uint64_t ldr, uint32_t inner,
                              const void *inner_weight, const void *inner_bias, const void *gate, uint32_t outer,
                              const void *outer_weight, const void *outer_bias, uint64_t rows, uint32_t hidden, float eps, float scale,
                              float residual_scale, double p, uint64_t seed, const int64_t *step, uint32_t type, uint32_t weight_type,
                              void *total, uint64_t ldt, void *y, uint64_t ldy, float *stats, nuq_stream_t stream)
{
    ResidualNormForward P{x, residual, inner_weight, inner_bias, gate, outer_weight, outer_bias, total, y, stats, {}, rows, ldx, ldr,
                          ldt, ldy, hidden, inner, outer, eps, 0.0f, residual_scale};
    if (!valid_seam(rows, hidden, type, weight_type, inner, outer, scale, residual_scale,
                    {inner_weight, inner_bias, gate, outer_weight, outer_bias}) || !draws_of(p, seed, step, P.draws) ||
        !std::isfinite(eps) || eps < 0.0f || (inner == NUQ_NO_NORM && (inner_weight || inner_bias)) ||
        (outer == NUQ_NO_NORM && (outer_weight || outer_bias || y)) || off_grid(stats, 4))
        return NUQ_EINVAL;
    if (rows == 0)
        return NUQ_OK;
    P.factor = scale * P.draws.keep;
    const uint32_t w = width(type);
    if (!valid_array(x, 1, w) || off_grid(residual, w) || !valid_array(total, 1, w) ||
        (outer != NUQ_NO_NORM && !valid_array(y, 1, w)) ||
        (rows > 1 && (ldt < hidden || (y && ldy < hidden) || other_stride(y, ldy, x, ldx) || other_stride(total, ldt, x, ldx) ||
                      other_stride(total, ldt, residual, ldr))))
        return NUQ_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return with_types(type, weight_type, [&](auto tt, auto wt) {
        using T = typename decltype(tt)::type;
        using W = typename decltype(wt)::type;
        const auto run = [&](auto team, auto elements, auto vec, auto many_c) {
            constexpr int TEAM = decltype(team)::value, E = decltype(elements)::value, VEC = decltype(vec)::value;
            const auto launch = [&](auto inner_c, auto once_c) {
                constexpr bool kInner = decltype(inner_c)::value, kMany = decltype(many_c)::value, kOnce = decltype(once_c)::value;
                constexpr uint32_t WG = kSeamForwardWG<TEAM, kMany>, TEAMS = WG / TEAM;
                const uint32_t most = resident_workgroups<k_residual_norm_forward<T, W, TEAM, E, VEC, kInner, kMany, kOnce>>(WG);
                if (!most)
                    return (int)NUQ_EHIP;
                const uint32_t grid = (uint32_t)std::min<uint64_t>((rows + TEAMS - 1) / TEAMS, most);
                hipLaunchKernelGGL((k_residual_norm_forward<T, W, TEAM, E, VEC, kInner, kMany, kOnce>), dim3(grid), dim3(WG), 0, st, P);
                return check_launch();
            };
            const auto with_inner = [&](auto once_c) {
                return inner != NUQ_NO_NORM ? launch(std::true_type{}, once_c) : launch(std::false_type{}, once_c);
            };
            return rows * hidden > kLastLevelCache / (4u * w) ? with_inner(std::true_type{}) : with_inner(std::false_type{});
        };
        if (hidden <= kManyColumns && rows * hidden > kManyElements)
            return with_seam_shape<T, SeamPass::kMany>(hidden, [&](auto team, auto elements, auto vec) {
                if constexpr (decltype(team)::value > 0)
                    return run(team, elements, vec, std::true_type{});
                else
                    return (int)NUQ_EINVAL;                  // (no such width)
            });
        return with_seam_shape<T, SeamPass::kFew>(hidden, [&](auto team, auto elements, auto vec) { return run(team, elements, vec, std::false_type{}); });
    });
}

uint64_t nuq_residual_norm_workspace_bytes(uint64_t rows, uint32_t hidden)
{
    return 4ull * kSeamSums * hidden * std::min<uint64_t>(rows, 1024u) + (hidden > kSumsInRegisters ? 8ull * rows : 0ull);
}

int nuq_residual_norm_backward(const void *dy, uint64_t ldg, const void *dtotal, uint64_t lda, const void *x, uint64_t ldx,
                               const void *total, uint64_t ldt, uint32_t inner, const void *inner_weight, const void *inner_bias,
                               const void *gate, uint32_t outer, const void *outer_weight, uint64_t rows, uint32_t hidden, float scale,
                               float residual_scale, double p, uint64_t seed, const int64_t *step, uint32_t type, uint32_t weight_type,
                               const float *stats, void *dx, uint64_t ldd, void *dresidual, uint64_t lde, void *dinner_weight,
                               void *dinner_bias, void *dgate, void *douter_weight, void *douter_bias, void *workspace,
                               uint64_t workspace_bytes, nuq_stream_t stream)
{
    ResidualNormBackward P{dy, dtotal, x, total, inner_weight, inner_bias, gate, outer_weight, stats, dx, dresidual,
                           static_cast<float *>(workspace), nullptr, {}, rows, ldg, lda, ldx, ldt, ldd, lde, hidden, inner, outer,
                           0.0f, residual_scale};
    const bool sums = dinner_weight || dinner_bias || dgate || douter_weight || douter_bias;
    if (!valid_seam(rows, hidden, type, weight_type, inner, outer, scale, residual_scale,
                    {inner_weight, inner_bias, gate, outer_weight, dinner_weight, dinner_bias, dgate, douter_weight, douter_bias}) ||
        !draws_of(p, seed, step, P.draws) ||
        (inner == NUQ_NO_NORM && (inner_weight || inner_bias || dinner_weight || dinner_bias)) ||
        (outer == NUQ_NO_NORM && (outer_weight || douter_weight || douter_bias || dy)))
        return NUQ_EINVAL;
    const uint32_t w = width(type);
    if (rows > 0 && (!valid_array(x, 1, w) || !valid_array(dx, 1, w) || !valid_array(stats, 1, 4) || off_grid(dtotal, w) ||
                     (outer != NUQ_NO_NORM ? !valid_array(dy, 1, w) || !valid_array(total, 1, w) : !dtotal) ||
                     off_grid(dresidual, w) ||
                     (rows > 1 && (ldd < hidden || (dresidual && lde < hidden) || other_stride(dx, ldd, dy, ldg) ||
                                   other_stride(dx, ldd, x, ldx) || other_stride(dresidual, lde, dtotal, lda) ||
                                   (outer != NUQ_NO_NORM && other_stride(dresidual, lde, total, ldt)))) ||
                     (sums && (!workspace || off_grid(workspace, 16)))))
        return NUQ_EINVAL;
    // wide rows: the sums are taken behind the rows' results, from what these must not have replaced
    if (rows > 0 && sums && hidden > kSumsInRegisters &&
        (dx == dy || dx == x || (dresidual && (dresidual == dtotal || dresidual == total))))
        return NUQ_EINVAL;
    if (rows > 0 && sums && workspace_bytes < nuq_residual_norm_workspace_bytes(rows, hidden))
        return NUQ_ECAPACITY;
    if (hidden > kSumsInRegisters && sums && outer != NUQ_NO_NORM)
        P.means = P.partial + (uint64_t)kSeamSums * hidden * std::min<uint64_t>(rows, 1024u);
    P.factor = scale * P.draws.keep;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return with_types(type, weight_type, [&](auto tt, auto wt) {
        using T = typename decltype(tt)::type;
        using W = typename decltype(wt)::type;
        uint32_t parts = 0;
        const int rc = rows == 0 ? (int)NUQ_OK : with_seam_shape<T, SeamPass::kBackward>(hidden, [&](auto team, auto elements, auto vec) {
            constexpr int TEAM = decltype(team)::value, E = decltype(elements)::value, VEC = decltype(vec)::value;
            constexpr uint32_t WG = kSeamBackwardWG<TEAM>, TEAMS = WG / TEAM;
            const auto run = [&](auto inner_c, auto sums_c, auto once_c) {
                constexpr bool kInner = decltype(inner_c)::value, kSums = decltype(sums_c)::value, kOnce = decltype(once_c)::value;
                const uint32_t most = resident_workgroups<k_residual_norm_backward<T, W, TEAM, E, VEC, kInner, kSums, kOnce>>(WG);
                if (!most)
                    return (int)NUQ_EHIP;
                parts = (uint32_t)std::min<uint64_t>((rows + TEAMS - 1) / TEAMS, kSums ? std::min(most, kSeamParts) : most);
                hipLaunchKernelGGL((k_residual_norm_backward<T, W, TEAM, E, VEC, kInner, kSums, kOnce>), dim3(parts), dim3(WG), 0, st, P);
                return check_launch();
            };
            const auto with_inner = [&](auto sums_c, auto once_c) {
                return inner != NUQ_NO_NORM ? run(std::true_type{}, sums_c, once_c) : run(std::false_type{}, sums_c, once_c);
            };
            if constexpr (TEAM * E <= (int)kSumsInRegisters) {
                if (!sums)
                    return with_inner(std::false_type{}, std::false_type{});
                return rows * hidden > kLastLevelCache / (6u * w) ? with_inner(std::true_type{}, std::true_type{})
                                                                  : with_inner(std::true_type{}, std::false_type{});
            } else {
                int done = with_inner(std::false_type{}, std::false_type{});     // (the sums read the rows again)
                if (done == NUQ_OK && sums) {
                    constexpr uint32_t COLUMNS = 256u * 16u / sizeof(T);
                    parts = (uint32_t)std::min<uint64_t>(rows, kWideParts);
                    hipLaunchKernelGGL((k_residual_norm_columns<T, W>), dim3((hidden + COLUMNS - 1u) / COLUMNS, parts), dim3(256), 0, st, P);
                    done = check_launch();
                }
                return done;
            }
        });
        if (rc != NUQ_OK || !sums)
            return rc;
        const SeamVectors V{inner_weight, inner_bias, gate, dinner_weight, dinner_bias, dgate, douter_weight, douter_bias, P.factor};
        hipLaunchKernelGGL((k_residual_norm_finish<W>), dim3((hidden + 15u) / 16u, 2), dim3(1024), 0, st, P.partial, parts,
                           hidden, V);
        return check_launch();
    });
}

}  // extern "C"
