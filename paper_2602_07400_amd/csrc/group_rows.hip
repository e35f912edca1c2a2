// Rows in the order of their groups (adapters), stable, with tables of tiles and chunks.
//
// A counting sort: rows are cut into runs, a block counts a run's rows of each group, the counts
// are summed up over runs and groups, and the block walks its run again, each wave its part of it
// 64 rows at a time: a row's place is its group's start, plus what earlier runs, waves and steps
// hold of the group, plus the equal rows before it in the step, which ballots give.  Rows keep
// their order within a group, so that sums over a group's rows do not depend on the schedule.
// Up to 4096 rows are one block's, one launch; more take three.
//
// What bounds it: chains of loads and LDS accesses, and fetching code that runs once: with 16
// steps of a wave unrolled, one block took 29 us for 12289 rows, in a loop 21.  2^18 rows of 24
// groups: 5, 8 and 9 us.
#include "adapters.h"

namespace bl {
namespace {

using namespace adapt;

// The place of this lane's row among the step's rows of its group, and how many those are:
// lanes of one group agree in every bit of its number, one ballot a bit.  (A ballot a group
// instead, 25 of them present: 32 us to place 2^18 rows, these 8.)
__device__ __forceinline__ void match(uint32_t group, bool valid, int bits, uint32_t &before,
                                      uint32_t &count)
{
    uint64_t same = __ballot(valid);
#pragma unroll 1
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot(group >> b & 1);
        same &= group >> b & 1 ? set : ~set;
    }
    before = __popcll(same & ((1ull << (threadIdx.x % kWave)) - 1));
    count = __popcll(same);
}

__device__ __forceinline__ int32_t group_of_row(const int32_t *ids, int64_t row, int32_t groups)
{
    const int32_t id = ids[row];
    return id >= 0 && id < groups ? id : groups;          // the last one: rows without a group
}

// A block's rows [lo, hi), at most 64 WAVES STEPS of them, a wave's part of them together.
// match_rows: counts [WAVES][all groups] of each wave's rows, and in seen a row's group and its
// place among its wave's.  place_rows: to the order, counts being places by now.
constexpr int kGroupBits = 13;
static_assert(kMaxGroups < 1 << kGroupBits, "a group and a place in 32 bits");

template <int WAVES, int STEPS>
__device__ __forceinline__ void match_rows(const int32_t *ids, int64_t lo, int64_t hi,
                                           int32_t groups, uint32_t *counts, uint32_t *seen)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int32_t all = groups + 1;
    const int bits = 32 - __builtin_clz(groups);          // (the number `groups` occurs too)
    uint32_t *mine = counts + wave * all;
    seen += wave * STEPS * kWave + lane;
    const int64_t first = lo + wave * STEPS * kWave + lane;
#pragma unroll
    for (int k = 0; k < STEPS; ++k)
        if (first + k * kWave < hi)
            seen[k * kWave] = (uint32_t)group_of_row(ids, first + k * kWave, groups);
    for (int32_t i = lane; i < all; i += kWave)
        mine[i] = 0;
    rows::wave_sync();
#pragma unroll 1
    for (int k = 0; k < STEPS && lo + (wave * STEPS + k) * kWave < hi; ++k) {
        const bool valid = first + k * kWave < hi;
        const uint32_t g = valid ? seen[k * kWave] : 0;
        uint32_t before, count;
        match(g, valid, bits, before, count);
        if (valid) {
            const uint32_t at = mine[g] + before;
            seen[k * kWave] = g | at << kGroupBits;
            __builtin_amdgcn_wave_barrier();
            if (before == 0)
                mine[g] = at + count;
        }
        rows::wave_sync();
    }
}

template <int WAVES, int STEPS>
__device__ __forceinline__ void place_rows(int64_t lo, int64_t hi, int32_t all,
                                           const uint32_t *counts, const uint32_t *seen,
                                           int32_t *order)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    seen += wave * STEPS * kWave + lane;
    const int64_t first = lo + wave * STEPS * kWave + lane;
#pragma unroll 2
    for (int k = 0; k < STEPS; ++k)
        if (first + k * kWave < hi) {
            const uint32_t s = seen[k * kWave], g = s & ((1u << kGroupBits) - 1);
            order[counts[wave * all + g] + (s >> kGroupBits)] = (int32_t)(first + k * kWave);
        }
}

// counts of a block's waves to places: from base [all groups] on, which is raised by what the
// block has.
template <int WAVES>
__device__ __forceinline__ void sum_waves(uint32_t *counts, uint32_t *base, int32_t all)
{
    for (int32_t i = threadIdx.x; i < all; i += kWave * WAVES) {
        uint32_t sum = base[i];
#pragma unroll 1
        for (int w = 0; w < WAVES; ++w) {
            const uint32_t own = counts[w * all + i];
            counts[w * all + i] = sum;
            sum += own;
        }
        base[i] = sum;
    }
}

// What sum_groups leaves, [all groups + 1] each: of rows, tiles, and the chunks and slots of
// both cuts.
constexpr int kSums = 6;
struct Starts {
    int32_t *of[kSums];
};

// The tables of tiles and chunks: eight lanes to a group's entries, and entries without a piece
// behind all of them.  A share of the groups and entries: those from `first` lanes on by `step`.
__device__ __forceinline__ void write_tables(const GroupArgs &a, const Starts &starts,
                                             int64_t first, int64_t step)
{
    const int32_t groups = a.groups + 1;
    const auto table = [&](Piece4 *to, int32_t size, const int32_t *pieces, const int32_t *slots,
                           int32_t g, int32_t lane) __attribute__((always_inline)) {
        const int32_t e0 = pieces[g], count = pieces[g + 1] - e0;
        const int32_t row0 = starts.of[0][g], rows = starts.of[0][g + 1] - row0;
        const int32_t slot0 = slots[g];
#pragma unroll 1
        for (int32_t k = lane; k < count; k += 8)
            to[e0 + k] = {g, row0 + k * size, min(size, rows - k * size), slot0 + k};
    };
#pragma unroll 1
    for (int64_t at = first; at < (int64_t)groups * 8; at += step) {
        const int32_t g = (int32_t)(at / 8), lane = (int32_t)(at % 8);
        table(a.tiles, kTile, starts.of[1], starts.of[1], g, lane);
        for (int c = 0; c < 2; ++c)
            table(a.cut[c].chunks, a.cut[c].rows, starts.of[2 + 2 * c], starts.of[3 + 2 * c], g,
                  lane);
    }
#pragma unroll 1
    for (int64_t e = starts.of[1][groups] + first; e < a.n_tiles; e += step)
        a.tiles[e] = {-1, 0, 0, 0};
    for (int c = 0; c < 2; ++c)
#pragma unroll 1
        for (int64_t e = starts.of[2 + 2 * c][groups] + first; e < a.cut[c].n; e += step)
            a.cut[c].chunks[e] = {-1, 0, 0, 0};
}

__device__ __forceinline__ Starts starts_of(const GroupArgs &a)
{
    return {{a.starts, a.tile_starts, a.cut[0].starts, a.cut[0].slots, a.cut[1].starts,
             a.cut[1].slots}};
}

// Exclusive sums over the groups' totals (in LDS), in one scan of six numbers, to the plan and to
// `near` [kSums][all groups + 1] in LDS, if that is no NULL.  A block of 64 * WAVES; part:
// kSums * WAVES words of LDS.
template <int WAVES>
__device__ __forceinline__ void sum_groups(const GroupArgs &a, const uint32_t *totals,
                                           int32_t *near, int32_t *part)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int32_t groups = a.groups + 1;
    const Starts to = starts_of(a);
    int32_t base[kSums] = {};
#pragma unroll 1
    for (int32_t g0 = 0; g0 < groups; g0 += kWave * WAVES) {
        const int32_t g = g0 + threadIdx.x;
        const int32_t rows = g < groups ? (int32_t)totals[g] : 0;
        int32_t v[kSums] = {rows, rows / kTile + (rows % kTile > 0)}, in[kSums];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int32_t chunks = rows / a.cut[c].rows + (rows % a.cut[c].rows > 0);
            v[2 + 2 * c] = chunks;
            v[3 + 2 * c] = chunks > 1 && g < a.groups ? chunks : 0;
        }
#pragma unroll
        for (int k = 0; k < kSums; ++k)
            in[k] = v[k];
#pragma unroll 1
        for (int d = 1; d < kWave; d *= 2)
#pragma unroll
            for (int k = 0; k < kSums; ++k) {
                const int32_t o = __shfl_up(in[k], d);
                in[k] += lane >= d ? o : 0;
            }
        if (lane == kWave - 1)
#pragma unroll
            for (int k = 0; k < kSums; ++k)
                part[k * WAVES + wave] = in[k];
        __syncthreads();
        int32_t all[kSums] = {}, before[kSums] = {};
#pragma unroll 1
        for (int w = 0; w < WAVES; ++w)
#pragma unroll
            for (int k = 0; k < kSums; ++k) {
                before[k] += w < wave ? part[k * WAVES + w] : 0;
                all[k] += part[k * WAVES + w];
            }
#pragma unroll
        for (int k = 0; k < kSums; ++k) {
            const int32_t start = base[k] + before[k] + in[k] - v[k];
            if (g < groups) {
                to.of[k][g] = start;
                if (near)
                    near[k * (groups + 1) + g] = start;
            }
            base[k] += all[k];
        }
        __syncthreads();
    }
    if (threadIdx.x == 0)
#pragma unroll
        for (int k = 0; k < kSums; ++k) {
            to.of[k][groups] = base[k];
            if (near)
                near[k * (groups + 1) + groups] = base[k];
        }
    __syncthreads();
}

// ---- one block ----
// LDS: a row's group and place, [WAVES][all groups] counts, [all groups] totals, starts
template <int WAVES, int STEPS>
__global__ __launch_bounds__(kWave * WAVES) void k_group_few(GroupArgs a)
{
    extern __shared__ uint32_t lds[];
    __shared__ int32_t part[kSums * WAVES];
    const int32_t all = a.groups + 1;
    uint32_t *seen = lds, *counts = lds + WAVES * STEPS * kWave, *base = counts + WAVES * all;
    int32_t *near = reinterpret_cast<int32_t *>(base + all);
    match_rows<WAVES, STEPS>(a.ids, 0, a.rows, a.groups, counts, seen);
    for (int32_t i = threadIdx.x; i < all; i += kWave * WAVES)
        base[i] = 0;
    __syncthreads();
    sum_waves<WAVES>(counts, base, all);
    __syncthreads();
    sum_groups<WAVES>(a, base, near, part);
    for (int32_t i = threadIdx.x; i < all * WAVES; i += kWave * WAVES)
        counts[i] += (uint32_t)near[i % all];
    __syncthreads();
    place_rows<WAVES, STEPS>(0, a.rows, all, counts, seen, a.order);
    Starts starts;
    for (int k = 0; k < kSums; ++k)
        starts.of[k] = near + k * (all + 1);
    write_tables(a, starts, threadIdx.x, kWave * WAVES);
}

// ---- many rows: a run a block ----
constexpr int kRunWaves = 4, kRunSteps = 4, kRunThreads = kRunWaves * kWave;
static_assert(kLeastRun == kRunThreads * kRunSteps, "a run is whole rounds of a block");

__global__ __launch_bounds__(kRunThreads) void k_group_count(GroupArgs a)
{
    extern __shared__ uint32_t lds[];
    const int32_t all = a.groups + 1;
    for (int32_t g = threadIdx.x; g < all; g += kRunThreads)
        lds[g] = 0;
    __syncthreads();
    const int64_t lo = blockIdx.x * a.run, hi = min(a.rows, lo + a.run);
#pragma unroll 4
    for (int64_t row = lo + threadIdx.x; row < hi; row += kRunThreads)
        atomicAdd(&lds[group_of_row(a.ids, row, a.groups)], 1u);
    __syncthreads();
    for (int32_t g = threadIdx.x; g < all; g += kRunThreads)
        a.counts[(int64_t)g * a.runs + blockIdx.x] = lds[g];
}

constexpr int kSumWaves = 16, kAhead = 4;                 // runs by the wave, loaded together
__global__ __launch_bounds__(kWave * kSumWaves) void k_group_sum(GroupArgs a)
{
    extern __shared__ uint32_t totals[];
    __shared__ int32_t part[kSums * kSumWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int32_t all = a.groups + 1;
#pragma unroll 1
    for (int32_t g = wave; g < all; g += kSumWaves) {     // a wave sums up a group's runs
        uint32_t base = 0;
        uint32_t *counts = a.counts + (int64_t)g * a.runs;
#pragma unroll 1
        for (int32_t r0 = 0; r0 < a.runs; r0 += kAhead * kWave) {
            uint32_t own[kAhead], in[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int32_t r = r0 + k * kWave + lane;
                in[k] = own[k] = r < a.runs ? counts[r] : 0;
            }
#pragma unroll 1
            for (int d = 1; d < kWave; d *= 2)
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const uint32_t o = __shfl_up(in[k], d);
                    in[k] += lane >= d ? o : 0;
                }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int32_t r = r0 + k * kWave + lane;
                if (r < a.runs)
                    counts[r] = base + in[k] - own[k];
                base += __shfl(in[k], kWave - 1);
            }
        }
        if (lane == 0)
            totals[g] = base;
    }
    __syncthreads();
    sum_groups<kSumWaves>(a, totals, nullptr, part);
}

__global__ __launch_bounds__(kRunThreads) void k_group_place(GroupArgs a)
{
    extern __shared__ uint32_t lds[];
    const int32_t all = a.groups + 1;
    if (blockIdx.x >= (uint32_t)a.runs) {                 // the tables, by blocks of their own
        write_tables(a, starts_of(a),
                     (int64_t)(blockIdx.x - a.runs) * kRunThreads + threadIdx.x,
                     (int64_t)(gridDim.x - a.runs) * kRunThreads);
        return;
    }
    uint32_t *seen = lds, *counts = lds + kLeastRun, *base = counts + kRunWaves * all;
    for (int32_t g = threadIdx.x; g < all; g += kRunThreads)
        base[g] = (uint32_t)a.starts[g] + a.counts[(int64_t)g * a.runs + blockIdx.x];
    const int64_t lo = blockIdx.x * a.run, hi = min(a.rows, lo + a.run);
#pragma unroll 1
    for (int64_t at = lo; at < hi; at += kLeastRun) {
        const int64_t end = min(hi, at + kLeastRun);
        match_rows<kRunWaves, kRunSteps>(a.ids, at, end, a.groups, counts, seen);
        __syncthreads();
        sum_waves<kRunWaves>(counts, base, all);
        __syncthreads();
        place_rows<kRunWaves, kRunSteps>(at, end, all, counts, seen, a.order);
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_group_rows(const int32_t *ids, int64_t rows, int32_t groups, void *plan,
                             hipStream_t stream)
{
    const GroupLayout l = group_layout(rows, groups);
    char *p = static_cast<char *>(plan);
    GroupArgs a;
    a.ids = ids;
    a.rows = rows;
    a.groups = groups;
    a.order = reinterpret_cast<int32_t *>(p + l.order);
    a.starts = reinterpret_cast<int32_t *>(p + l.starts);
    a.tile_starts = reinterpret_cast<int32_t *>(p + l.tile_starts);
    a.tiles = reinterpret_cast<Piece4 *>(p + l.tiles);
    for (int c = 0; c < 2; ++c)
        a.cut[c] = {reinterpret_cast<Piece4 *>(p + l.cut[c].chunks),
                    reinterpret_cast<int32_t *>(p + l.cut[c].starts),
                    reinterpret_cast<int32_t *>(p + l.cut[c].slots), l.cut[c].n, l.cut[c].rows};
    a.counts = reinterpret_cast<uint32_t *>(p + l.counts);
    a.n_tiles = l.n_tiles;
    a.run = l.run;
    a.runs = l.runs;
    const size_t all = (size_t)groups + 1;
    // one block up to 4096 rows (16 steps a wave, 12289 rows: 21 us; three launches 13)
    const auto few = [&](auto waves, auto steps) {
        constexpr int W = decltype(waves)::value, S = decltype(steps)::value;
        hipLaunchKernelGGL((k_group_few<W, S>), dim3(1), dim3(W * kWave),
                           (W * S * kWave + (W + 1 + kSums) * all + kSums) * 4, stream, a);
        return hipGetLastError();
    };
    using std::integral_constant;
    if (all <= 512 && rows <= 16 * kWave)
        return few(integral_constant<int, 16>(), integral_constant<int, 1>());
    if (all <= 512 && rows <= 16 * 4 * kWave)
        return few(integral_constant<int, 16>(), integral_constant<int, 4>());
    hipLaunchKernelGGL(k_group_count, dim3(l.runs), dim3(kRunThreads), all * 4, stream, a);
    hipLaunchKernelGGL(k_group_sum, dim3(1), dim3(kWave * kSumWaves), all * 4, stream,
                       a);
    const uint32_t tables = (uint32_t)std::min<int64_t>(64, (l.n_tiles + kRunThreads - 1) / kRunThreads);
    hipLaunchKernelGGL(k_group_place, dim3(l.runs + tables), dim3(kRunThreads),
                       (kLeastRun + (kRunWaves + 1) * all) * 4, stream, a);
    return hipGetLastError();
}

}  // namespace bl
