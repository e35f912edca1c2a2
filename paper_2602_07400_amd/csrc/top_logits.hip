// Top logits: the k largest logits of every row with their classes, and the row's
// log-normalizer log sum_i e^(l_i / T): what a teacher hands on to a student.
//
// One pass over the row, as it arrives, takes the running maximum and sum of the
// softmax and every lane's largest logit.  The classes >= lo, the k-th largest of the
// lanes', are k or a few more: they go to a list in LDS that is put in order.  Where
// the bound does not hold so few (k near the number of lanes or above), counts of keys
// in ever narrower intervals raise it; where no bound does (many equal logits), tau, the
// k-th largest key, is what they end at, and the list gets the classes above tau and the
// first ones equal to it.  (Groups of less than a wave find tau by bisection.)  Entries
// (key, class) are unique, so the order in which the list fills does not matter.
//
// What bounds it: long rows, the exponentials and unpacking (about 9 instructions an
// element; the VALU is active in 76 of 100 cycles) beside the read: 2048 x 131072 bf16,
// k 64, 105 us, 5.1 TB/s of the 7.0 that a plain read reaches (161 with the row kept in registers and one block a CU, 646 with
// bisection over the row); single rows, the block's chain of barriers: 1 x 50021
// float32, k 256, 21 us; many short rows, see k_top_lanes.
#include "logit_rows.h"

namespace bl {
namespace {

using namespace rows;

struct TopArgs {
    const char *logits;
    int64_t stride;            // bytes from row to row
    int64_t n_rows;
    int32_t n, k;
    float inv_t;
    char *values;              // [rows][k], the logits' type
    int32_t *indices;          // [rows][k]
    float *log_norm;           // [rows] or NULL
};

template <int TYPE>
struct TopRows : TopArgs {
    void skip(int64_t rows)
    {
        logits += rows * stride;
        values += rows * k * Elem<TYPE>::kBytes;
        indices += rows * k;
        if (log_norm)
            log_norm += rows;
    }
};

template <int TYPE, class L>
__global__ __launch_bounds__(L::kBlock, L::G == kWave ? 4 : 8) void k_top(TopArgs a)
{
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    typedef Piece<TYPE, L::VEC> P;
    constexpr int G = L::G;
    __shared__ Scratch scratch;
    __shared__ uint64_t lists[L::kGroups][L::kList];
    __shared__ uint64_t placed[L::kGroups][L::kCounted];
    __shared__ uint32_t fills[L::kGroups];
    const int gi = group_of<G>();
    const int64_t r = (int64_t)blockIdx.x * L::kGroups + gi;
    if (r >= a.n_rows)
        return;
    Group<G> g(threadIdx.x - gi * G, &scratch);
    uint64_t *list = lists[gi];
    uint32_t *fill = &fills[gi];
    const char *src = a.logits + r * a.stride;
    Row<TYPE, G, L::NV, L::VEC, L::RESIDENT, (G < kWave)> row(src, a.n, g.t);

    const float c = a.inv_t * kLog2e;
    Softmax<TYPE, !L::RESIDENT> sm;
    Cmp top = E::lowest(), most[L::NV];                   // the lane's and its pieces' largest
    static_for<L::NV>([&](auto j) __attribute__((always_inline)) { most[j] = E::lowest(); });
    row.each([&](auto j, int32_t, const P &p) {
        Cmp vm = E::lowest();
#pragma unroll
        for (int u = 0; u < L::VEC; ++u)
            vm = Max()(vm, p.get(u));                     // (a NaN never is)
        top = Max()(top, vm);
        if constexpr (L::RESIDENT)
            most[j] = vm;
        if (a.log_norm) {
            // (the select changes nothing but the compiler's registers: without it more of
            // them are spilled around the list, 2048 x 131072 in 122 us instead of 106)
            sm.raise(vm > E::lowest() ? vm : E::lowest(), c);
            const Cmp from = sm.from();
            float part = sm.start();
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                part += __builtin_amdgcn_exp2f(E::minus(p.get(u), from) * c);
            sm.add(part);
        }
    });
    if (a.log_norm) {
        if (!(sm.s >= 0.0f)) {                            // a NaN, or +inf - inf: without them
            sm.s = sm.lost = 0.0f;
            row.stream([&](int32_t, const P &p) {
                float part = sm.start();
#pragma unroll
                for (int u = 0; u < L::VEC; ++u) {
                    const float e = E::minus(p.get(u), sm.m);
                    part += e <= 0.0f ? __builtin_amdgcn_exp2f(e * c) : 0.0f;
                }
                sm.add(part);
            });
        }
        sm = combine(g, sm, c);
        if (g.t == 0)
            a.log_norm[r] = sm.log_norm(a.inv_t);
    }

    uint32_t lo = E::kFirstKey, found = 0xFFFFFFFFu, k = a.k;
    if constexpr (G >= kWave) {
        // k lanes each have a logit >= lo; all of the row's classes are where fewer
        // lanes have any
        if (k <= (uint32_t)G)
            lo = max(lo, group_mth(g, top > E::lowest() ? E::key(top) : 0, k, (uint32_t *)list));
        found = collect<TYPE, L>(g, row, most, E::from_key(lo), list, fill);
    }
    if (found > (uint32_t)L::kList) {
        // the k-th key, or a range of keys around it that fits the list
        Range<uint32_t> at = {lo, E::key(g.reduce(top, Max())) + 1, 0, found};
        if constexpr (G > kWave) {
            at = narrow<TYPE, L, uint32_t>(g, row, most, at, k, L::kList, (uint32_t *)list,
                                           [](Cmp) { return 1u; });
            if (at.before + at.here <= (uint32_t)L::kList)
                found = collect<TYPE, L>(g, row, most, E::from_key(at.lo), list, fill);
        }
        if constexpr (G < kWave) {
            const auto count_from = [&](Cmp v) __attribute__((always_inline)) {
                uint32_t count = 0;
                row.each([&](auto, int32_t, const P &p) {
#pragma unroll
                    for (int u = 0; u < L::VEC; ++u)
                        count += p.get(u) >= v;
                });
                return g.reduce(count, Add());
            };
            k = min(k, count_from(E::from_key(at.lo)));
            while (k && at.hi - at.lo > 1) {              // count(>= lo) >= k > count(>= hi)
                const uint32_t mid = at.lo + (at.hi - at.lo) / 2;
                if (count_from(E::from_key(mid)) >= k)
                    at.lo = mid;
                else
                    at.hi = mid;
            }
        }
        if (found > (uint32_t)L::kList) {
            // those above it, then the first classes of the equal ones
            const Cmp tau = E::from_key(at.lo);
            g.barrier();
            if (g.t == 0)
                *fill = 0;
            g.barrier();
            row.stream([&](int32_t i, const P &p) {
#pragma unroll
                for (int u = 0; u < L::VEC; ++u) {
                    const Cmp v = p.get(u);
                    if (k && v > tau)
                        list[atomicAdd(fill, 1u)] = entry(E::key(v), i + u);
                }
            });
            g.barrier();
            found = *fill;
            row.stream([&](int32_t i, const P &p) {
                if (found >= k)
                    return;
                uint32_t mine = 0, total;
#pragma unroll
                for (int u = 0; u < L::VEC; ++u)
                    mine += p.get(u) == tau;
                uint32_t place = found + g.scan(mine, total);
                found += total;
#pragma unroll
                for (int u = 0; u < L::VEC; ++u)
                    if (p.get(u) == tau) {
                        if (place < k)
                            list[place] = entry(at.lo, i + u);
                        ++place;
                    }
            });
            found = k;
            g.barrier();
        }
    }
    k = min(k, found);

    // the list in order
    if (found <= (uint32_t)L::kCounted) {
        place_entries(g, list, found, placed[gi], nullptr, [](uint64_t) { return 0.0f; });
        list = placed[gi];
    } else if constexpr (G >= kWave) {
        sort_entries(g, list, found);
    }
    char *values = a.values + r * a.k * E::kBytes;
    int32_t *indices = a.indices + r * a.k;
    const auto put = [&](uint32_t to, int32_t cls, Cmp v) {
        if (TYPE != kI32 && v == 0)
            v = load_one<TYPE>(src, cls);                 // with its sign
        indices[to] = cls;
        if constexpr (E::kBytes == 4)
            reinterpret_cast<Cmp *>(values)[to] = v;
        else if constexpr (TYPE == kF16)
            reinterpret_cast<_Float16 *>(values)[to] = (_Float16)v;
        else
            reinterpret_cast<uint16_t *>(values)[to] = __float_as_uint(v) >> 16;
    };
    for (uint32_t e = g.t; e < k; e += G)
        put(e, class_of(list[e]), E::from_key(key_of(list[e])));
    for (uint32_t e = k + g.t; e < (uint32_t)a.k; e += G)
        put(e, -1, E::lowest());
}

// The larger and the smaller of two positive doubles (plain v_max and v_min: the
// compiler's own put a canonicalization before each).
__device__ __forceinline__ double max_of(double a, double b)
{
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ double min_of(double a, double b)
{
    double r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// A lane a row, k <= K: every class is carried down a sorted list in registers.  Class
// and key are the mantissa of a double (52 bits: 32 of key, then the class reversed), so
// that a step of the list is one maximum and one minimum.  262144 x 100 int32, k 10: 92
// us (216 with a group of 32 lanes a row and bisection).  What bounds it is how few waves
// there are to take turns: 26 KB of LDS each leave a CU 4.3 of them on average, and the
// VALU is active in 40 of 100 cycles (24 of some 40 instructions a class in the list).
template <int TYPE, int K>
__global__ __launch_bounds__(kWave) void k_top_lanes(TopArgs a)
{
    typedef Elem<TYPE == kI32 ? kI32 : kF32> E;           // (the tile's elements)
    typedef typename E::Cmp Cmp;
    extern __shared__ uint32_t tile[];
    const int64_t r0 = (int64_t)blockIdx.x * kWave;
    const int32_t rows = (int32_t)min((int64_t)kWave, a.n_rows - r0);
    load_tile<TYPE>(a.logits + r0 * a.stride, a.stride, rows, a.n, a.n | 1, tile);
    wave_sync();
    const uint32_t *own = tile + min((int32_t)threadIdx.x, rows - 1) * (a.n | 1);
    const auto at = [&](int i) __attribute__((always_inline)) {
        Cmp v;
        __builtin_memcpy(&v, &own[i], 4);
        return v;
    };
    constexpr uint32_t kOne = 0x43300000u;                // 2^52
    double best[K];
#pragma unroll
    for (int j = 0; j < K; ++j)
        best[j] = __hiloint2double(kOne, 0);
#pragma unroll 4
    for (int i = 0; i < a.n; ++i) {
        const Cmp v = at(i);
        const uint32_t key = v > E::lowest() ? E::key(v) : 0;
        double x = __hiloint2double(kOne | key >> 12, key << 20 | (kLaneClasses - 1 - i));
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const double down = min_of(best[j], x);
            best[j] = max_of(best[j], x);
            x = down;
        }
    }
    const auto key_at = [&](int j) __attribute__((always_inline)) {
        return (uint32_t)__double2hiint(best[j]) << 12 | (uint32_t)__double2loint(best[j]) >> 20;
    };
    if (a.log_norm) {
        const uint32_t first = key_at(0);
        const float c = a.inv_t * kLog2e;
        Softmax<TYPE == kI32 ? kI32 : kF32> sm;
        if (first)
            sm.m = E::from_key(first);
#pragma unroll 4
        for (int i = 0; i < a.n; ++i) {
            const Cmp v = at(i);
            sm.s += v > E::lowest() ? __builtin_amdgcn_exp2f(E::minus(v, sm.m) * c) : 0.0f;
        }
        if ((int32_t)threadIdx.x < rows)
            a.log_norm[r0 + threadIdx.x] = sm.log_norm(a.inv_t);
    }
    // the lists by way of the tile, to be stored in whole lines
    uint32_t value[K];
    int32_t cls[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        cls[j] = key_at(j) ? kLaneClasses - 1 - (int32_t)(__double2loint(best[j]) & 0xFFFFF) : -1;
        const Cmp none = E::lowest();
        __builtin_memcpy(&value[j], &none, 4);
        if (j < a.k && cls[j] >= 0)
            value[j] = own[cls[j]];
    }
    wave_sync();
    const int32_t half = kWave * a.k;
#pragma unroll
    for (int j = 0; j < K; ++j)
        if (j < a.k) {
            tile[threadIdx.x * a.k + j] = value[j];
            tile[half + threadIdx.x * a.k + j] = (uint32_t)cls[j];
        }
    wave_sync();
    for (int32_t e = threadIdx.x; e < rows * a.k; e += kWave) {
        const int64_t to = r0 * a.k + e;
        a.indices[to] = (int32_t)tile[half + e];
        const uint32_t v = tile[e];
        if constexpr (TYPE == kF16)
            reinterpret_cast<_Float16 *>(a.values)[to] = (_Float16)__uint_as_float(v);
        else if constexpr (TYPE == kBf16)
            reinterpret_cast<uint16_t *>(a.values)[to] = (uint16_t)(v >> 16);
        else
            reinterpret_cast<uint32_t *>(a.values)[to] = v;
    }
}

template <int TYPE>
hipError_t launch_lanes(const TopArgs &a, hipStream_t stream)
{
    const uint32_t blocks = (uint32_t)((a.n_rows + kWave - 1) / kWave);
    const size_t words = (size_t)kWave * ((a.n | 1) > 2 * a.k ? a.n | 1 : 2 * a.k);
    if (a.k <= 4)
        k_top_lanes<TYPE, 4><<<blocks, kWave, words * 4, stream>>>(a);
    else if (a.k <= 8)
        k_top_lanes<TYPE, 8><<<blocks, kWave, words * 4, stream>>>(a);
    else
        k_top_lanes<TYPE, 12><<<blocks, kWave, words * 4, stream>>>(a);
    return hipGetLastError();
}

// Rows that go to lanes: a lane's time grows with a row's classes, a group's with the
// number of rows.  float32, k 10, lanes against groups in us:
//   rows       4096       8192      16384      32768      65536     262144
//   10 cl.   5.6, 8.3   5.6, 8.2   5.4, 8.5  5.9, 10.5  6.2, 16.5  10.6, 49
//   37      10.7, 9.4  10.7, 9.6  10.8, 11.8 11.7, 18.8 12.0, 31.5  23, 107
//   100     22.8, 10.4 23.0, 12.8 23.0, 20.3 24.9, 34.4 26.0, 62.4  87, 231
//   128     27.5, 10.4 27.7, 13.0 27.8, 20.6 30.4, 35.0 31.1, 64.0 133, 236
// (at 128 x 32768 bfloat16 31, 28).
constexpr int64_t kLaneRowsAClass = 256;
// Entries a lane's list has room for.  Lists of 16 and 24 entries, which are not built,
// take 99 and 121 us at 262144 x 100 float32, groups 234 and 250.
constexpr int32_t kLaneEntries = 12;

}  // namespace

hipError_t launch_top_logits(const void *logits, int32_t type, int64_t n_rows, int32_t n,
                             int64_t row_stride, int32_t k, float inv_t, void *values,
                             int32_t *indices, float *log_norm, hipStream_t stream)
{
    return with_type(type, [&](auto ty) {
        constexpr int TYPE = decltype(ty)::value;
        const TopArgs a = {static_cast<const char *>(logits), row_stride * Elem<TYPE>::kBytes,
                           n_rows, n, k, inv_t, static_cast<char *>(values), indices, log_norm};
        if (n <= kLaneClasses && k <= kLaneEntries && n_rows >= kLaneRowsAClass * n)
            return launch_lanes<TYPE>(a, stream);
        return with_layout<TYPE>(n, 0, [&](auto layout) {
            typedef decltype(layout) L;
            return in_launches(TopRows<TYPE>{a}, L::kBlock, L::kGroups,
                               [&](const TopArgs &part, uint32_t blocks) {
                k_top<TYPE, L><<<blocks, L::kBlock, 0, stream>>>(part);
            });
        });
    });
}

}  // namespace bl
