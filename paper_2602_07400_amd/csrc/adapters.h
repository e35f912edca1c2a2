// Low-rank adapters (internal): what the plan of grouped rows holds, and the arguments of the
// kernels.
#pragma once

#include <algorithm>

#include "logit_rows.h"

namespace bl {
namespace adapt {

using rows::kBf16;
using rows::kF16;
using rows::kF32;
using rows::kI32;

constexpr int kTile = 64;               // rows of a tile, all of one group
constexpr int32_t kMaxGroups = 4096;    // (a wave's counters in LDS)
constexpr int32_t kMaxRank = 128;
constexpr int32_t kMaxRuns = 1024;
constexpr int64_t kLeastRun = 1024;     // rows that a block sorts at a time

// Rows [first, first + count) of the order, of one group (-1: no piece).  slot: of a group of
// several chunks, the chunk's partial sums in the workspace.
struct Piece4 {
    int32_t group, first, count, slot;
};

// ---- the plan: rows by group ----
// Gradients of the weights are partial sums over chunks of a group's rows.  The plan has the
// chunks of two cuts: small ones give narrow adapters blocks enough, large ones keep the
// partial sums of wide adapters few.
struct CutLayout {
    size_t chunks, starts, slots;
    int64_t n, n_slots;
    int32_t rows;
};
struct GroupLayout {
    size_t order, starts, tile_starts, tiles, counts, bytes;
    CutLayout cut[2];
    int64_t n_tiles, run;
    int32_t runs;
};

inline GroupLayout group_layout(int64_t n_rows, int32_t groups)
{
    GroupLayout l;
    const int64_t small = std::max<int64_t>(256, n_rows / 1024 / kTile * kTile);
    l.n_tiles = n_rows / kTile + groups + 1;              // at most a partial one a group
    l.run = std::max<int64_t>(1, (n_rows + kMaxRuns * kLeastRun - 1) / (kMaxRuns * kLeastRun)) *
            kLeastRun;
    l.runs = (int32_t)((n_rows + l.run - 1) / l.run);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const size_t all = (size_t)groups + 2;
    l.order = take((size_t)n_rows * 4);
    l.starts = take(all * 4);
    l.tile_starts = take(all * 4);
    l.tiles = take((size_t)l.n_tiles * sizeof(Piece4));
    for (int c = 0; c < 2; ++c) {
        CutLayout &k = l.cut[c];
        k.rows = (int32_t)(c ? 4 * small : small);
        k.n = n_rows / k.rows + groups + 1;
        k.n_slots = 2 * (n_rows / k.rows);                // k > 1 chunks: over (k - 1) rows rows
        k.chunks = take((size_t)k.n * sizeof(Piece4));
        k.starts = take(all * 4);
        k.slots = take(all * 4);
    }
    l.counts = take((size_t)l.runs * (groups + 1) * 4);
    l.bytes = at;
    return l;
}

struct Cut {
    Piece4 *chunks;
    int32_t *starts, *slots;
    int64_t n;
    int32_t rows;
};
struct GroupArgs {
    const int32_t *ids;
    int64_t rows, n_tiles, run;
    int32_t groups, runs;
    int32_t *order, *starts, *tile_starts;
    Piece4 *tiles;
    Cut cut[2];
    uint32_t *counts;
};

// ---- a pass through adapters ----
// Forward: out = base_scale base + scale up (down x), hidden = down x.  Back: the same with
// x the gradient of out, down^T and up^T in each other's places, and no base.
struct PassArgs {
    const char *x;
    int64_t x_stride;                   // strides in bytes from row to row
    const char *w1, *w2;                // forward: down [rank][k], up [m][rank];
                                        // back: up [k][rank], down [rank][m]
    int64_t w1_step, w2_step;           // bytes from adapter to adapter
    int32_t k, m, rank, groups;
    const float *scales;                // [groups] or NULL
    float scale;
    const char *base;                   // or NULL
    int64_t base_stride;
    int32_t base_i32;
    float base_scale;
    char *out;                          // or NULL: hidden alone
    int64_t out_stride;
    float *hidden;                      // [rows][rank] or NULL
    // rows by a plan, or (tiles NULL) a tile each by their ids
    const Piece4 *tiles;
    const int32_t *order, *ids;
    int64_t n_rows, n_tiles;
    // wide adapters: h by parts [splits][n_rows][rank] (hidden itself, if that is one part);
    // splits 0: narrow ones, in one kernel
    float *partial;
    int32_t splits;
};

// Whether a plan's rows go through one kernel, a tile and its adapter a block: rows of x and of
// out of at most 512 bytes each, and 64 KB of LDS (2^17 rows, 100 -> 100: rank 8 float32 45 us, by
// wide kernels 64; rank 64 bfloat16 56 and 68; 64 rows 10 and 14).
template <int W> bool fits_narrow(int32_t k, int32_t m, int32_t rank, bool back);

// Parts of the k terms of wide adapters: for about 768 blocks (8192 rows, 4096 -> 4096, rank 64:
// 84 us, 87 with 1024, 92 with 1536), whose waves (8 or, above rank
// 32, 4) have a unit of 128 bytes or more each.
inline int32_t split_terms(int64_t n_tiles, int32_t k, int32_t rank, int32_t el_bytes)
{
    const int64_t share = (rank <= 32 ? 8 : 4) * 128;
    const int64_t most = ((int64_t)k * el_bytes + share - 1) / share;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>({most, 8, 768 / n_tiles}));
}

struct PassLayout {
    bool narrow;
    int64_t n_tiles;
    int32_t splits;
    size_t bytes;                       // of partial
};
inline PassLayout pass_layout(int64_t n_rows, int32_t groups, int32_t rank, int32_t k,
                              int32_t el_bytes, bool planned, bool narrow)
{
    PassLayout l;
    l.n_tiles = planned ? group_layout(n_rows, groups).n_tiles : n_rows;
    l.narrow = planned && narrow;
    l.splits = l.narrow || n_rows == 0
                   ? 0 : split_terms(planned ? l.n_tiles * (kTile / 32) : n_rows, k, rank,
                                     el_bytes);
    l.bytes = (size_t)l.splits * n_rows * rank * 4;
    return l;
}

// Blocks of a tile in the second product of wide adapters: about 1024 in all, with at most eight
// units of columns each (128 bytes, back 256).  (Four, eight, sixteen units: 200 rows of 48
// adapters, 4096 -> 12288, 36, 34 and 40 us; 8192 rows, 4096 -> 4096, 82, 83 and 85.)
inline int32_t expand_blocks(const PassArgs &a, int32_t el_bytes, bool back)
{
    const int64_t unit = back ? 256 : 128;
    const int64_t units = a.out ? ((int64_t)a.m * el_bytes + unit - 1) / unit : 1;
    return (int32_t)std::min<int64_t>(units,
                                      std::max<int64_t>((units + 7) / 8, 1024 / a.n_tiles));
}

// Whether each launch of a pass stays below 2^32 lanes.
inline bool fits_launches(const PassArgs &a, int32_t el_bytes, bool back)
{
    return a.n_tiles * std::max(expand_blocks(a, el_bytes, back), 4 * a.splits) < 1 << 24;
}

// Gradients: d down [groups][rank][n_in] = sum scale back x^T, d up [groups][n_out][rank] =
// sum scale grad hidden^T, over a group's rows.
struct GradJob {
    const char *y;                      // rows of x, or of the gradient of out
    int64_t y_stride;
    int32_t y_i32, cols, blocks;        // columns, and blocks of them
    const float *h;                     // [rows][rank]: back, or hidden
    char *out;                          // or NULL: no such job
    int32_t transposed;                 // out [cols][rank] instead of [rank][cols]
    float *partial;                     // [slots][rank][cols]
};
struct GradArgs {
    GradJob job[2];
    const Piece4 *chunks;
    const int32_t *order, *chunk_starts, *slot_starts;   // (chunk_starts NULL: no rows)
    int64_t n_chunks;
    int32_t rank, groups;
    const float *scales;
    float scale;
};

template <int W> hipError_t launch_pass(const PassArgs &a, bool x_i32, bool back,
                                        hipStream_t stream);
template <int W> hipError_t launch_grads(const GradArgs &a, hipStream_t stream);
// columns that a block of launch_grads takes
template <int W> int32_t grad_block();

}  // namespace adapt
}  // namespace bl
