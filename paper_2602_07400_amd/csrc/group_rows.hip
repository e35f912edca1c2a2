// Rows in the order of their groups (adapters), stable, with tables of tiles and chunks.
//
// A counting sort: rows are cut into runs, a wave counts a run's rows of each group, the
// counts are summed up over runs and groups, and the wave walks its run again, 64 rows at a
// time: a row's place is its group's start, plus what earlier runs and steps hold of the
// group, plus the equal rows before it in the step, which a ballot gives.  Rows keep their
// order within a group, so that sums over a group's rows do not depend on the schedule.
// Few rows are done by one block with its counters in LDS (one launch), more by three
// launches.  What bounds it: the launches and a wave's chain of steps, not the 8 bytes a row.
#include "adapters.h"

namespace bl {
namespace {

using namespace adapt;

// The place of this lane's row among the step's rows of its group, and how many those are:
// lanes of one group agree in every bit of its number, one ballot a bit (a ballot a group
// instead, 25 of them present: 32 us for 2^18 rows in runs of 1024, these 9).
__device__ __forceinline__ void match(uint32_t group, bool valid, int bits, uint32_t &before,
                                      uint32_t &count)
{
    uint64_t same = __ballot(valid);
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

// The last of `starts` [count + 1] (ascending, starts[0] = 0) at or below `at`.
template <class P>
__device__ __forceinline__ int32_t find(P starts, int32_t count, int32_t at)
{
    int32_t lo = 0, hi = count;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) / 2;
        if (starts[mid] <= at)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// Entries of a table of pieces of `size` rows, for the indexes from `first` on by `step`.
template <class P>
__device__ __forceinline__ void write_pieces(Piece4 *table, int64_t entries, int32_t size,
                                             P piece_starts, P starts, P slot_starts,
                                             int32_t groups, int64_t first, int64_t step)
{
    const int32_t used = piece_starts[groups];
    for (int64_t e = first; e < entries; e += step) {
        Piece4 p = {-1, 0, 0, 0};
        if (e < used) {
            const int32_t g = find(piece_starts, groups, (int32_t)e);
            const int32_t k = (int32_t)e - piece_starts[g], from = starts[g] + k * size;
            p = {g, from, min(size, starts[g + 1] - from), slot_starts[g] + k};
        }
        table[e] = p;
    }
}

// Exclusive sums over the groups' totals: rows, tiles, and the chunks and slots of both cuts.
// A block of 64 * WAVES; part: kSums * WAVES words of LDS.
constexpr int kSums = 6;
template <int WAVES>
__device__ void sum_groups(const GroupArgs &a, int32_t *part)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int32_t groups = a.groups + 1;
    int32_t *const to[kSums] = {a.starts,         a.tile_starts,  a.cut[0].starts,
                                a.cut[0].slots, a.cut[1].starts, a.cut[1].slots};
    int32_t base[kSums] = {};
    for (int32_t g0 = 0; g0 < groups; g0 += kWave * WAVES) {
        const int32_t g = g0 + threadIdx.x;
        const int32_t rows = g < groups ? (int32_t)a.totals[g] : 0;
        int32_t v[kSums] = {rows, rows / kTile + (rows % kTile > 0)}, in[kSums];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int32_t chunks = rows / a.cut[c].rows + (rows % a.cut[c].rows > 0);
            v[2 + 2 * c] = chunks;
            v[3 + 2 * c] = chunks > 1 && g < a.groups ? chunks : 0;
        }
#pragma unroll
        for (int k = 0; k < kSums; ++k) {
            in[k] = v[k];
            for (int d = 1; d < kWave; d *= 2) {
                const int32_t o = __shfl_up(in[k], d);
                if (lane >= d)
                    in[k] += o;
            }
            if (lane == kWave - 1)
                part[k * WAVES + wave] = in[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSums; ++k) {
            int32_t all = 0, before = 0;
            for (int w = 0; w < WAVES; ++w) {
                before += w < wave ? part[k * WAVES + w] : 0;
                all += part[k * WAVES + w];
            }
            if (g < groups)
                to[k][g] = base[k] + before + in[k] - v[k];
            base[k] += all;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0)
#pragma unroll
        for (int k = 0; k < kSums; ++k)
            to[k][groups] = base[k];
    __syncthreads();
}

// A run's rows [lo, hi) to their places; next: the places of the run's next row of each group.
// The ids of kAhead steps are loaded together.
constexpr int kAhead = 4;
template <class P>
__device__ __forceinline__ void place_rows(const int32_t *ids, int64_t lo, int64_t hi,
                                           int32_t groups, P next, int32_t *order)
{
    const int bits = 32 - __builtin_clz(groups);          // (the number `groups` occurs too)
    for (int64_t at = lo; at < hi; at += kAhead * kWave) {
        uint32_t g[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t row = at + k * kWave + threadIdx.x % kWave;
            g[k] = row < hi ? (uint32_t)group_of_row(ids, row, groups) : 0;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t row = at + k * kWave + threadIdx.x % kWave;
            const bool valid = row < hi;
            uint32_t before, count;
            match(g[k], valid, bits, before, count);
            uint32_t to = 0;
            if (valid)
                to = next[g[k]];
            __builtin_amdgcn_wave_barrier();
            if (valid) {
                order[to + before] = (int32_t)row;
                if (before == 0)
                    next[g[k]] = to + count;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// ---- one block ----
template <int WAVES>
__global__ __launch_bounds__(kWave * WAVES) void k_group_few(GroupArgs a)
{
    extern __shared__ uint32_t counts[];                  // [WAVES][all groups]
    __shared__ int32_t part[kSums * WAVES];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int32_t all = a.groups + 1;
    uint32_t *mine = counts + wave * all;
    for (int32_t i = threadIdx.x; i < WAVES * all; i += kWave * WAVES)
        counts[i] = 0;
    __syncthreads();
    const int64_t run = (a.rows + kWave * WAVES - 1) / (kWave * WAVES) * kWave;
    const int64_t lo = min(a.rows, wave * run), hi = min(a.rows, lo + run);
#pragma unroll 4
    for (int64_t row = lo + lane; row < hi; row += kWave)
        atomicAdd(&mine[group_of_row(a.ids, row, a.groups)], 1u);
    __syncthreads();
    for (int32_t g = threadIdx.x; g < all; g += kWave * WAVES) {
        uint32_t sum = 0;
        for (int w = 0; w < WAVES; ++w) {
            const uint32_t own = counts[w * all + g];
            counts[w * all + g] = sum;
            sum += own;
        }
        a.totals[g] = sum;
    }
    __syncthreads();
    sum_groups<WAVES>(a, part);
    for (int32_t i = threadIdx.x; i < WAVES * all; i += kWave * WAVES)
        counts[i] += (uint32_t)a.starts[i % all];
    __syncthreads();
    place_rows(a.ids, lo, hi, a.groups, mine, a.order);
    write_pieces(a.tiles, a.n_tiles, kTile, a.tile_starts, a.starts, a.starts, all, threadIdx.x,
                 kWave * WAVES);
    for (int c = 0; c < 2; ++c)
        write_pieces(a.cut[c].chunks, a.cut[c].n, a.cut[c].rows, a.cut[c].starts, a.starts,
                     a.cut[c].slots, all, threadIdx.x, kWave * WAVES);
}

// ---- many rows ----
__global__ __launch_bounds__(kWave) void k_group_count(GroupArgs a)
{
    extern __shared__ uint32_t counts[];
    const int32_t all = a.groups + 1;
    for (int32_t g = threadIdx.x; g < all; g += kWave)
        counts[g] = 0;
    __syncthreads();
    const int64_t lo = blockIdx.x * a.run, hi = min(a.rows, lo + a.run);
#pragma unroll 4
    for (int64_t row = lo + threadIdx.x; row < hi; row += kWave)
        atomicAdd(&counts[group_of_row(a.ids, row, a.groups)], 1u);
    __syncthreads();
    for (int32_t g = threadIdx.x; g < all; g += kWave)
        a.counts[(int64_t)g * a.runs + blockIdx.x] = counts[g];
}

constexpr int kSumWaves = 16;
__global__ __launch_bounds__(kWave * kSumWaves) void k_group_sum(GroupArgs a)
{
    __shared__ int32_t part[kSums * kSumWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int32_t all = a.groups + 1;
    for (int32_t g = wave; g < all; g += kSumWaves) {     // a wave sums up a group's runs
        uint32_t base = 0;
        for (int32_t r0 = 0; r0 < a.runs; r0 += kWave) {
            const int32_t r = r0 + lane;
            uint32_t *at = a.counts + (int64_t)g * a.runs + r;
            const uint32_t own = r < a.runs ? *at : 0;
            uint32_t in = own;
            for (int d = 1; d < kWave; d *= 2) {
                const uint32_t o = __shfl_up(in, d);
                if (lane >= d)
                    in += o;
            }
            if (r < a.runs)
                *at = base + in - own;
            base += __shfl(in, kWave - 1);
        }
        if (lane == 0)
            a.totals[g] = base;
    }
    __syncthreads();
    sum_groups<kSumWaves>(a, part);
}

__global__ __launch_bounds__(kWave) void k_group_place(GroupArgs a)
{
    extern __shared__ uint32_t next[];
    const int32_t all = a.groups + 1;
    for (int32_t g = threadIdx.x; g < all; g += kWave)
        next[g] = (uint32_t)a.starts[g] + a.counts[(int64_t)g * a.runs + blockIdx.x];
    __syncthreads();
    const int64_t lo = blockIdx.x * a.run, hi = min(a.rows, lo + a.run);
    place_rows(a.ids, lo, hi, a.groups, next, a.order);
    const int64_t first = (int64_t)blockIdx.x * kWave + threadIdx.x,
                  step = (int64_t)gridDim.x * kWave;
    write_pieces(a.tiles, a.n_tiles, kTile, a.tile_starts, a.starts, a.starts, all, first, step);
    for (int c = 0; c < 2; ++c)
        write_pieces(a.cut[c].chunks, a.cut[c].n, a.cut[c].rows, a.cut[c].starts, a.starts,
                     a.cut[c].slots, all, first, step);
}

// One block up to here.
constexpr int64_t kFewRows = 16384;

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
    a.totals = reinterpret_cast<uint32_t *>(p + l.totals);
    a.counts = reinterpret_cast<uint32_t *>(p + l.counts);
    a.n_tiles = l.n_tiles;
    a.run = l.run;
    a.runs = l.runs;
    const size_t all = (size_t)groups + 1;
    if (rows <= kFewRows) {
        // (a block's 64 KB of counters: groups that are many leave it fewer waves)
        if (all <= 1024)
            hipLaunchKernelGGL(k_group_few<16>, dim3(1), dim3(16 * kWave), 16 * all * 4, stream,
                               a);
        else
            hipLaunchKernelGGL(k_group_few<3>, dim3(1), dim3(3 * kWave), 3 * all * 4, stream, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(k_group_count, dim3(l.runs), dim3(kWave), all * 4, stream, a);
    hipLaunchKernelGGL(k_group_sum, dim3(1), dim3(kWave * kSumWaves), 0, stream, a);
    hipLaunchKernelGGL(k_group_place, dim3(l.runs), dim3(kWave), all * 4, stream, a);
    return hipGetLastError();
}

}  // namespace bl
