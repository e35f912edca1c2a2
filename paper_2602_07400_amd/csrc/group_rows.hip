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
// one ballot a group that is present.
__device__ __forceinline__ void match(int32_t group, bool valid, uint32_t &before,
                                      uint32_t &count)
{
    uint64_t left = __ballot(valid);
    const uint64_t mine = 1ull << (threadIdx.x % kWave);
    before = count = 0;
    while (left) {
        const int32_t one = __shfl(group, __builtin_ctzll(left));
        const uint64_t same = __ballot(valid && group == one);
        if (valid && group == one) {
            before = __popcll(same & (mine - 1));
            count = __popcll(same);
        }
        left &= ~same;
    }
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

// Exclusive sums over the groups' totals: rows, tiles, chunks and slots.  A block of
// 64 * WAVES; part: 4 * WAVES words of LDS.
template <int WAVES>
__device__ void sum_groups(const GroupArgs &a, int32_t *part)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int32_t groups = a.groups + 1;
    int32_t *const to[4] = {a.starts, a.tile_starts, a.chunk_starts, a.slot_starts};
    int32_t base[4] = {0, 0, 0, 0};
    for (int32_t g0 = 0; g0 < groups; g0 += kWave * WAVES) {
        const int32_t g = g0 + threadIdx.x;
        const int32_t rows = g < groups ? (int32_t)a.totals[g] : 0;
        const int32_t chunks = rows / a.chunk + (rows % a.chunk > 0);
        const int32_t v[4] = {rows, rows / kTile + (rows % kTile > 0), chunks,
                              chunks > 1 && g < a.groups ? chunks : 0};
        int32_t in[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
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
        for (int k = 0; k < 4; ++k) {
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
        for (int k = 0; k < 4; ++k)
            to[k][groups] = base[k];
    __syncthreads();
}

// A run's rows [lo, hi) to their places; next: the places of the run's next row of each group.
template <class P>
__device__ __forceinline__ void place_rows(const int32_t *ids, int64_t lo, int64_t hi,
                                           int32_t groups, P next, int32_t *order)
{
    for (int64_t at = lo; at < hi; at += kWave) {
        const int64_t row = at + threadIdx.x % kWave;
        const bool valid = row < hi;
        const int32_t g = valid ? group_of_row(ids, row, groups) : 0;
        uint32_t before, count;
        match(g, valid, before, count);
        uint32_t to = 0;
        if (valid)
            to = next[g];
        __builtin_amdgcn_wave_barrier();
        if (valid) {
            order[to + before] = (int32_t)row;
            if (before == 0)
                next[g] = to + count;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- one block ----
template <int WAVES>
__global__ __launch_bounds__(kWave * WAVES) void k_group_few(GroupArgs a)
{
    extern __shared__ uint32_t counts[];                  // [WAVES][all groups]
    __shared__ int32_t part[4 * WAVES];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int32_t all = a.groups + 1;
    uint32_t *mine = counts + wave * all;
    for (int32_t i = threadIdx.x; i < WAVES * all; i += kWave * WAVES)
        counts[i] = 0;
    __syncthreads();
    const int64_t run = (a.rows + kWave * WAVES - 1) / (kWave * WAVES) * kWave;
    const int64_t lo = min(a.rows, wave * run), hi = min(a.rows, lo + run);
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
    write_pieces(a.tiles, a.n_tiles, kTile, a.tile_starts, a.starts, a.slot_starts, all, threadIdx.x,
                 kWave * WAVES);
    write_pieces(a.chunks, a.n_chunks, a.chunk, a.chunk_starts, a.starts, a.slot_starts, all, threadIdx.x,
                 kWave * WAVES);
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
    for (int64_t row = lo + threadIdx.x; row < hi; row += kWave)
        atomicAdd(&counts[group_of_row(a.ids, row, a.groups)], 1u);
    __syncthreads();
    for (int32_t g = threadIdx.x; g < all; g += kWave)
        a.counts[(int64_t)g * a.runs + blockIdx.x] = counts[g];
}

constexpr int kSumWaves = 16;
__global__ __launch_bounds__(kWave * kSumWaves) void k_group_sum(GroupArgs a)
{
    __shared__ int32_t part[4 * kSumWaves];
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
    write_pieces(a.tiles, a.n_tiles, kTile, a.tile_starts, a.starts, a.slot_starts, all, first, step);
    write_pieces(a.chunks, a.n_chunks, a.chunk, a.chunk_starts, a.starts, a.slot_starts, all, first, step);
}

// One block up to here: a wave's steps of 64 rows are a chain of about 0.3 us each.
constexpr int64_t kFewRows = 8192;

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
    a.chunk_starts = reinterpret_cast<int32_t *>(p + l.chunk_starts);
    a.slot_starts = reinterpret_cast<int32_t *>(p + l.slot_starts);
    a.tiles = reinterpret_cast<Piece4 *>(p + l.tiles);
    a.chunks = reinterpret_cast<Piece4 *>(p + l.chunks);
    a.totals = reinterpret_cast<uint32_t *>(p + l.totals);
    a.counts = reinterpret_cast<uint32_t *>(p + l.counts);
    a.n_tiles = l.n_tiles;
    a.n_chunks = l.n_chunks;
    a.chunk = l.chunk;
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
