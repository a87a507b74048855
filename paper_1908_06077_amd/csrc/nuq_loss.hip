// C ABI of softmax cross entropy over a large vocabulary (see include/nuq.h): argument checks, the workspace, pieces of the vocabulary
// and launches.  A source file of its own, so that it is built beside the others.
#include "../../include/nuq.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "nuq_loss_kernels.hpp"
#include "nuq_train_host.hpp"

namespace {

using namespace nuq;

constexpr uint32_t kMostLossRows = 1u << 20, kMostHidden = 1u << 16, kMostVocab = 1u << 24;

uint64_t up(uint64_t n, uint64_t m) { return (n + m - 1) / m * m; }
uint32_t over(uint64_t n, uint64_t m) { return (uint32_t)((n + m - 1) / m); }

struct LossShape {
    const void *x, *w;
    uint64_t ldx, ldw;
    uint32_t rows, hidden, vocab, type;

    bool valid(uint64_t all_rows) const
    {
        return all_rows <= kMostLossRows && hidden >= 1 && hidden <= kMostHidden && vocab >= 1 && vocab <= kMostVocab && type <= NUQ_F16 &&
               (uint64_t)rows * vocab <= 1ull << 38;
    }
    uint32_t bytes() const { return width(type); }
    // Whether loads of 16 bytes take the rows as they stand.  (Rows that overlap are laid out anew: what a tile may read is reckoned by its
    // rows' stride.)
    bool whole(const void *p, uint64_t ld) const
    {
        return !off_grid(p, 16) && ld >= hidden && ld * bytes() % 16u == 0 && hidden * bytes() % 16u == 0 && ld * bytes() < 1u << 22;
    }
    bool pack_x() const { return !whole(x, ldx); }
    bool pack_w() const { return !whole(w, ldw); }
    uint64_t packed() const { return up(hidden, 64); }       // elements of a packed row
};

// Parts of a workspace one after the other, each at a multiple of 256 bytes.
struct Parts {
    char *base;
    uint64_t used = 0;
    template <class T>
    T *take(uint64_t n)
    {
        T *const p = reinterpret_cast<T *>(base + used);
        used = up(used + n * sizeof(T), 256);
        return p;
    }
};

// Tiles.  Up to 64 rows a product passes its other operand by: tiles of all rows, with more stages.  Else the tile whose rounds of 256
// workgroups take the least, counted in rounds of 256 x 256: a round of 128 x 128, a quarter of the work, counts 0.35 in 16 bits (0.3 was
// tried: gradients of 1003 rows of 1001 against 10007 weights in fp16 took 128 us, with the one round of 256 x 256 that 0.35 chooses 119),
// one of 64 x 64 counts 0.11.  fp32 products take eight times as long and hide what smaller tiles read: no 256 x 256 there.  Against one
// rule by the number of rows: 1341 x 1189 against 3799 weights in bfloat16 forward 36 us instead of 46, gradients of 13209 x 259 against
// 1127 in bfloat16 204 instead of 316.
enum class TileSize { k32, k64Rows, k64, k128, k256 };
TileSize tile_for(uint64_t columns, uint64_t rows, uint32_t bytes, bool with_64)
{
    if (rows <= 32)
        return TileSize::k32;
    if (rows <= 64)
        return TileSize::k64Rows;
    const auto rounds = [&](uint64_t size) { return (double)(((columns + size - 1) / size * ((rows + size - 1) / size) + 255u) / 256u); };
    const double t256 = bytes == 2 ? rounds(256) : 1e30, t128 = rounds(128) * (bytes == 2 ? 0.35 : 0.25),
                 t64 = with_64 ? rounds(64) * (bytes == 2 ? 0.11 : 0.07) : 1e30;
    return t256 <= t128 && t256 <= t64 ? TileSize::k256 : t128 <= t64 ? TileSize::k128 : TileSize::k64;
}
uint32_t tile_columns(TileSize t) { return t == TileSize::k256 ? 256 : t == TileSize::k64 ? 64 : 128; }
uint32_t tile_rows(TileSize t) { return t == TileSize::k256 ? 256 : t == TileSize::k128 ? 128 : t == TileSize::k32 ? 32 : 64; }

// f(Type<tile>).  kWith64: tiles of 64 x 64 may be asked for; kFew: those of few rows.
template <class T, bool kAcrossA, bool kAcrossB, bool kFew, bool kWith64, class F>
int with_tile(TileSize t, F &&f)
{
    if constexpr (sizeof(T) == 2)
        if (t == TileSize::k256)
            return f(Type<ProductTile<T, 256, 256, 2, 4, 2, kAcrossA, kAcrossB>>{});
    if constexpr (kFew) {
        if (t == TileSize::k32)
            return f(Type<ProductTile<T, 128, 32, 4, 1, 4, kAcrossA, kAcrossB>>{});
        if (t == TileSize::k64Rows)
            return f(Type<ProductTile<T, 128, 64, 4, 1, 3, kAcrossA, kAcrossB>>{});
    }
    if constexpr (kWith64)
        if (t == TileSize::k64)
            return f(Type<ProductTile<T, 64, 64, 2, 2, 4, kAcrossA, kAcrossB>>{});
    return f(Type<ProductTile<T, 128, 128, 2, 2, 2, kAcrossA, kAcrossB>>{});
}

// Each product's: the logits forward, the logits backward, the weights' gradient (its rows are the vocabulary's), the rows' gradient
// (which is split over the vocabulary where its tiles are few, so they may be large).
// Forward the smallest only where those of 128 x 128 leave half the CUs idle: their parts of the vocabulary take twice the workspace.
// (656 x 1756 against 504 in fp32 115 -> 41 us, 361 x 2743 against 317 in fp16 47 -> 30.)  The rows' gradient in fp32 takes them where a row
// fits one: 6818 x 37 against 28141 1262 -> 935 us.
TileSize logits_tile(const LossShape &S) { return tile_for(S.vocab, S.rows, S.bytes(), (uint64_t)over(S.vocab, 128) * over(S.rows, 128) <= 128u); }
TileSize gradient_tile(const LossShape &S, uint32_t piece) { return tile_for(piece, S.rows, S.bytes(), true); }
TileSize weights_tile(const LossShape &S, uint32_t piece)
{
    // (fp32, whose tiles take long: small ones where those of 128 x 128 leave half the CUs idle.  Gradients of 6321 x 905 against 1414 weights,
    // 96 tiles, 725 -> 553 us; of 6818 x 37 against 28141, whose pieces have fewer still, 2083 -> 1253)
    if (S.bytes() == 4 && (uint64_t)over(S.hidden, 128) * over(piece, 128) <= 128u)
        return TileSize::k64;
    return tile_for(S.hidden, std::max(piece, 65u), S.bytes(), false);
}
TileSize rows_tile(const LossShape &S)
{
    return S.rows <= 32 ? TileSize::k32 : S.rows <= 64 ? TileSize::k64Rows : S.bytes() == 4 ? (S.hidden <= 64 ? TileSize::k64 : TileSize::k128)
                                                                           : S.rows > 128 && S.hidden > 128 ? TileSize::k256 : TileSize::k128;
}

struct ForwardParts {
    char *x, *w;
    float2 *part;
    float *sums, *of_target, *row_loss;
    uint32_t groups;
    uint64_t used;
    ForwardParts(const LossShape &S, void *workspace, bool smooth)
    {
        Parts P{static_cast<char *>(workspace)};
        x = P.take<char>(S.pack_x() ? S.rows * S.packed() * S.bytes() : 0);
        w = P.take<char>(S.pack_w() ? S.vocab * S.packed() * S.bytes() : 0);
        groups = over(S.vocab, tile_columns(logits_tile(S)));
        part = P.take<float2>((uint64_t)groups * S.rows);
        sums = P.take<float>(smooth ? (uint64_t)groups * S.rows : 0);
        of_target = P.take<float>(S.rows);
        row_loss = P.take<float>(S.rows);
        used = P.used;
    }
};

// How many ways a product whose tiles leave CUs idle splits its depth (`steps` of it): as many workgroups as fill whole rounds of 256,
// three hundredths of the time for another set of sums to write and add.
uint32_t splits_of(uint64_t tiles, uint32_t steps, uint32_t most_splits)
{
    uint32_t best = 1;
    double most = 0.0;
    for (uint32_t s = 1; s <= std::max(1u, std::min(most_splits, steps / 8u)); ++s) {
        const double used = (double)(tiles * s) / (double)((tiles * s + 255u) / 256u * 256u) / (1.0 + 0.03 * (s - 1));
        if (used > most * 1.001) {
            most = used;
            best = s;
        }
    }
    return best;
}

// Entries of the vocabulary whose d is in the workspace at a time: at most 320 MiB of them (2048 at least), and of those numbers the one
// whose three products take the fewest steps of rounds of 256 tiles.
uint32_t piece_of(const LossShape &S)
{
    const uint64_t row = (uint64_t)S.rows * S.bytes(), most = std::min<uint64_t>(std::max<uint64_t>((320ull << 20) / row, 2048u), 1u << 20) / 256u;
    const uint64_t all = over(S.vocab, 256);
    if (all <= most)
        return (uint32_t)up(S.vocab, 64);
    const uint64_t nt = over(S.rows, 256), ht = over(S.hidden, 256), depth = 128 / S.bytes();
    const auto rounds = [](uint64_t tiles) { return (tiles + 255u) / 256u; };
    const auto steps = [&](uint64_t tiles) {                 // of a piece of so many tiles
        return rounds(tiles * nt) * (over(S.hidden, depth) + 3u) + rounds(tiles * ht) * over(S.rows, depth) + rounds(ht * nt) * tiles * 256u / depth;
    };
    uint64_t best = most, least = ~0ull;
    for (uint64_t tiles = most; tiles >= std::max<uint64_t>(most / 2u, 8u); --tiles) {
        const uint64_t cost = all / tiles * steps(tiles) + (all % tiles ? steps(all % tiles) : 0u);
        if (cost < least) {
            least = cost;
            best = tiles;
        }
    }
    return (uint32_t)(best * 256u);
}

struct BackwardParts {
    char *x, *w, *d, *clean;
    int32_t *code;
    float *factor, *scale, *largest, *sums;
    uint32_t piece, splits, each;
    uint64_t ld_sums, used;
    BackwardParts(const LossShape &S, void *workspace)
    {
        Parts P{static_cast<char *>(workspace)};
        const uint64_t b = S.bytes();
        piece = piece_of(S);
        const uint64_t wide = up(piece, 64);
        x = P.take<char>(S.pack_x() ? S.rows * S.packed() * b : 0);
        w = P.take<char>(S.pack_w() ? S.vocab * S.packed() * b : 0);
        code = P.take<int32_t>(S.rows);
        factor = P.take<float>(S.rows);
        scale = P.take<float>(S.rows);
        largest = P.take<float>(1);
        clean = P.take<char>(S.rows * S.packed() * b);
        d = P.take<char>(S.rows * wide * b);
        // for more than one set of sums: as much as d and the weights take
        const uint64_t more = std::max<uint64_t>(4ull << 20, S.rows * wide * b + (uint64_t)S.vocab * S.hidden * b);
        const uint32_t depth = 128u / (uint32_t)b, steps = over(wide, depth);
        splits = splits_of((uint64_t)over(S.hidden, tile_columns(rows_tile(S))) * over(S.rows, tile_rows(rows_tile(S))), steps,
                           1u + (uint32_t)std::min<uint64_t>(63u, more / (4u * S.rows * up(S.hidden, 4))));
        each = over(steps, splits) * depth;
        ld_sums = up(S.hidden, 4);
        sums = P.take<float>(splits * S.rows * ld_sums);
        used = P.used;
    }
};

template <class T>
int pack(const void *from, uint64_t ld, uint64_t rows, uint32_t columns, char *to, uint64_t to_ld, const int32_t *code, const float *factor,
         hipStream_t st)
{
    const uint64_t vectors = rows * (to_ld * sizeof(T) / 16u);
    hipLaunchKernelGGL(k_loss_pack<T>, dim3((uint32_t)std::min<uint64_t>((vectors + 255u) / 256u, 16384u)), dim3(256), 0, st,
                       static_cast<const T *>(from), ld, rows, columns, reinterpret_cast<T *>(to), (uint32_t)to_ld, code, factor);
    return check_launch();
}

// The rows and weights as the products take them: packed into the workspace where they do not stand so.
template <class T>
int operands(const LossShape &S, char *x, char *w, LossOperands &O, hipStream_t st)
{
    O = {S.x, S.w, (uint32_t)(S.ldx * sizeof(T)), (uint32_t)(S.ldw * sizeof(T)), over((uint64_t)S.hidden * sizeof(T), 16), S.rows, S.vocab, 0, 0};
    if (S.pack_x()) {
        if (const int rc = pack<T>(S.x, S.ldx, S.rows, S.hidden, x, S.packed(), nullptr, nullptr, st); rc != NUQ_OK)
            return rc;
        O.x = x;
        O.stride_x = (uint32_t)(S.packed() * sizeof(T));
    }
    if (S.pack_w()) {
        if (const int rc = pack<T>(S.w, S.ldw, S.vocab, S.hidden, w, S.packed(), nullptr, nullptr, st); rc != NUQ_OK)
            return rc;
        O.w = w;
        O.stride_w = (uint32_t)(S.packed() * sizeof(T));
    }
    return NUQ_OK;
}

bool valid_loss(const LossShape &S, uint64_t rows, const int64_t *target, float smoothing, const float *lse, const void *workspace)
{
    if (!S.valid(rows) || !(smoothing >= 0.0f && smoothing < 1.0f) || !valid_array(S.w, 1, S.bytes()))
        return false;
    return rows == 0 || (valid_array(S.x, 1, S.bytes()) && valid_array(target, 1, 8) && valid_array(lse, 1, 4) &&
                         valid_array(workspace, 1, 16));
}

}  // namespace

extern "C" {

uint64_t nuq_linear_cross_entropy_workspace_bytes(const void *x, uint64_t ldx, const void *weight, uint64_t ldw, uint64_t rows,
                                                  uint32_t hidden, uint32_t vocab, uint32_t type, int backward)
{
    const LossShape S{x, weight, ldx, ldw, (uint32_t)rows, hidden, vocab, type};
    if (!S.valid(rows) || rows == 0)
        return 0;
    return backward ? BackwardParts(S, nullptr).used : ForwardParts(S, nullptr, true).used;
}

int nuq_linear_cross_entropy_forward(const void *x, uint64_t ldx, const void *weight, uint64_t ldw, uint64_t rows, uint32_t hidden,
                                     uint32_t vocab, uint32_t type, const int64_t *target, int64_t ignore, float smoothing, float *loss,
                                     float *lse, float *mean, void *workspace, uint64_t workspace_bytes, nuq_stream_t stream)
{
    const LossShape S{x, weight, ldx, ldw, (uint32_t)rows, hidden, vocab, type};
    if (!valid_loss(S, rows, target, smoothing, lse, workspace) || off_grid(loss, 4) || off_grid(mean, 4))
        return NUQ_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    LossJoin J{target, nullptr, nullptr, nullptr, loss, lse, mean, flags_ptr(), ignore, S.rows, vocab, 0, smoothing};
    if (!J.flags)
        return NUQ_EHIP;
    if (rows == 0) {
        if (mean)
            hipLaunchKernelGGL(k_loss_mean, dim3(1), dim3(1024), 0, st, J);
        return check_launch();
    }
    const bool smooth = smoothing > 0.0f;
    const ForwardParts W(S, workspace, smooth);
    if (workspace_bytes < W.used)
        return NUQ_ECAPACITY;
    int rc = with_type(type, [&](auto tt) {
        using T = typename decltype(tt)::type;
        LossForward P{{}, target, W.part, W.sums, W.of_target};
        if (const int done = operands<T>(S, W.x, W.w, P.O, st); done != NUQ_OK)
            return done;
        return with_tile<T, false, false, true, true>(logits_tile(S), [&](auto tile) {
            using Tile = typename decltype(tile)::type;
            P.O.mt = over(vocab, Tile::BM);
            P.O.nt = over(rows, Tile::BN);
            const auto run = [&](auto smooth_c) {
                constexpr bool kSmooth = decltype(smooth_c)::value;
                const uint32_t most = resident_workgroups<k_loss_logits<T, Tile, kSmooth>>(Tile::THREADS);
                if (!most)
                    return (int)NUQ_EHIP;
                hipLaunchKernelGGL((k_loss_logits<T, Tile, kSmooth>), dim3(std::min(P.O.mt * P.O.nt, most)), dim3(Tile::THREADS), 0, st, P);
                return check_launch();
            };
            return smooth ? run(std::true_type{}) : run(std::false_type{});
        });
    });
    if (rc != NUQ_OK)
        return rc;
    J.part = W.part;
    J.sums = smooth ? W.sums : nullptr;
    J.of_target = W.of_target;
    J.row_loss = loss ? loss : W.row_loss;
    J.groups = W.groups;
    if (rows <= 16) {
        if (rows == 1)
            hipLaunchKernelGGL((k_loss_join<1, true>), dim3(1), dim3(1024), 0, st, J);
        else
            hipLaunchKernelGGL((k_loss_join<16, true>), dim3(1), dim3(1024), 0, st, J);
        return check_launch();
    }
    hipLaunchKernelGGL((k_loss_join<16, false>), dim3(over(rows, 16)), dim3(1024), 0, st, J);
    if (mean)
        hipLaunchKernelGGL(k_loss_mean, dim3(1), dim3(1024), 0, st, J);
    return check_launch();
}

int nuq_linear_cross_entropy_backward(const void *x, uint64_t ldx, const void *weight, uint64_t ldw, uint64_t rows, uint32_t hidden,
                                      uint32_t vocab, uint32_t type, const int64_t *target, int64_t ignore, float smoothing,
                                      const float *lse, const float *grad, int grad_per_row, const float *mean, void *dx, uint64_t ldd,
                                      void *dweight, uint64_t lde, void *workspace, uint64_t workspace_bytes, nuq_stream_t stream)
{
    const LossShape S{x, weight, ldx, ldw, (uint32_t)rows, hidden, vocab, type};
    const uint32_t b = width(type);
    if (!valid_loss(S, rows, target, smoothing, lse, workspace) || (rows > 0 && !valid_array(grad, 1, 4)) || off_grid(mean, 4) ||
        off_grid(dx, b) || off_grid(dweight, b) || (dx && rows > 1 && ldd < hidden) || (dweight && vocab > 1 && lde < hidden))
        return NUQ_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    LossRows R{target, grad, mean, nullptr, nullptr, nullptr, nullptr, flags_ptr(), ignore, S.rows, vocab,
               grad_per_row != 0, type == NUQ_F16 ? 1.0f / kGradientScale<_Float16> : 1.0f};
    if (!R.flags)
        return NUQ_EHIP;
    if (rows == 0)                                           // sums over no rows
        return !dweight ? (int)NUQ_OK : with_type(type, [&](auto tt) {
            using T = typename decltype(tt)::type;
            using Tile = ProductTile<T, 128, 128, 2, 2, 2, true, true>;
            LossProduct P{weight, weight, 16, 16, 0, 0, 0, 0, 0, hidden, vocab, over(hidden, Tile::BM), over(vocab, Tile::BN), dweight, lde, 0, nullptr};
            hipLaunchKernelGGL((k_loss_product<T, Tile, T, true, false>), dim3(P.mt * P.nt), dim3(Tile::THREADS), 0, st, P);
            return check_launch();
        });
    const BackwardParts W(S, workspace);
    if (workspace_bytes < W.used)
        return NUQ_ECAPACITY;
    if (!dx && !dweight)
        return NUQ_OK;
    R.code = W.code;
    R.factor = W.factor;
    R.scale = W.scale;
    R.largest = W.largest;
    hipLaunchKernelGGL(k_loss_rows, dim3(grad_per_row ? 1u : over(rows, 1024)), dim3(1024), 0, st, R);
    if (const int rc = check_launch(); rc != NUQ_OK)
        return rc;
    return with_type(type, [&](auto tt) {
        using T = typename decltype(tt)::type;
        constexpr uint32_t VEC = 16u / sizeof(T);
        LossGradient G{{}, W.code, lse, W.d, 0, 0, smoothing / (float)vocab, 1.0f - smoothing};
        int rc = operands<T>(S, W.x, W.w, G.O, st);
        if (rc == NUQ_OK && dweight)
            rc = pack<T>(x, ldx, rows, hidden, W.clean, S.packed(), W.code, W.factor, st);
        const char *const all = static_cast<const char *>(G.O.w);
        for (uint32_t first = 0; rc == NUQ_OK && first < vocab; first += W.piece) {
            const uint32_t here = std::min(W.piece, vocab - first);
            G.first = first;
            G.O.w = all + (uint64_t)first * G.O.stride_w;
            G.O.vocab = here;
            G.padded_vocab = (uint32_t)up(here, 64);
            const uint32_t stride_d = G.padded_vocab * (uint32_t)sizeof(T);
            rc = with_tile<T, false, false, true, true>(gradient_tile(S, here), [&](auto tile) {
                using Tile = typename decltype(tile)::type;
                G.O.mt = over(here, Tile::BM);
                G.O.nt = over(rows, Tile::BN);
                const uint32_t most = resident_workgroups<k_loss_gradient<T, Tile>>(Tile::THREADS);
                if (!most)
                    return (int)NUQ_EHIP;
                hipLaunchKernelGGL((k_loss_gradient<T, Tile>), dim3(std::min(G.O.mt * G.O.nt, most)), dim3(Tile::THREADS), 0, st, G);
                return check_launch();
            });
            if (rc == NUQ_OK && dweight)
                rc = with_tile<T, true, true, false, sizeof(T) == 4>(weights_tile(S, here), [&](auto tile) {
                    using Tile = typename decltype(tile)::type;
                    LossProduct P{W.clean, W.d, (uint32_t)(S.packed() * sizeof(T)), stride_d, (uint32_t)S.packed() / VEC, G.padded_vocab / VEC,
                                  S.rows, S.rows, (uint32_t)up(rows, 64), hidden, here, over(hidden, Tile::BM), over(here, Tile::BN),
                                  static_cast<T *>(dweight) + first * lde, lde, 0, W.largest};
                    hipLaunchKernelGGL((k_loss_product<T, Tile, T, true, false>), dim3(P.mt * P.nt), dim3(Tile::THREADS), 0, st, P);
                    return check_launch();
                });
            if (rc == NUQ_OK && dx)
                rc = with_tile<T, true, false, true, sizeof(T) == 4>(rows_tile(S), [&](auto tile) {
                    using Tile = typename decltype(tile)::type;
                    LossProduct P{G.O.w, W.d, G.O.stride_w, stride_d, S.pack_w() ? (uint32_t)S.packed() / VEC : hidden / VEC, 0, here,
                                  G.padded_vocab, W.each, hidden, S.rows, over(hidden, Tile::BM), over(rows, Tile::BN), W.sums, W.ld_sums,
                                  rows * W.ld_sums, nullptr};
                    const dim3 grid(P.mt * P.nt * W.splits);
                    if (first)
                        hipLaunchKernelGGL((k_loss_product<T, Tile, float, false, true>), grid, dim3(Tile::THREADS), 0, st, P);
                    else
                        hipLaunchKernelGGL((k_loss_product<T, Tile, float, false, false>), grid, dim3(Tile::THREADS), 0, st, P);
                    return check_launch();
                });
        }
        if (rc == NUQ_OK && dx) {
            const uint64_t vectors = rows * over(hidden, 4);
            hipLaunchKernelGGL(k_loss_rows_gradient<T>, dim3((uint32_t)std::min<uint64_t>((vectors + 255u) / 256u, 16384u)), dim3(256), 0, st,
                               W.sums, W.ld_sums, rows * W.ld_sums, W.splits, W.code, W.scale, S.rows, hidden, static_cast<T *>(dx), ldd);
            rc = check_launch();
        }
        return rc;
    });
}

}  // extern "C"
