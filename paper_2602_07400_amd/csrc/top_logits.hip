// Top logits: the k largest logits of every row with their classes, and the row's
// log-normalizer log sum_i e^(l_i / T): what a teacher hands on to a student.
//
// One pass over the row takes the running maximum and sum of the softmax.  The k-th
// largest key tau is then found by bisection on counts (key >= tau), the classes
// above tau and the first classes equal to it fill a list in LDS, and each entry's
// place is the number of entries before it.  Keys (key, class) are unique, so the
// order in which the list fills does not matter.
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

template <int TYPE, class L>
__global__ __launch_bounds__(L::kBlock) void k_top(TopArgs a)
{
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    extern __shared__ uint64_t lists[];                   // [rows of the block][min(k, n)]
    __shared__ Scratch scratch;
    __shared__ uint32_t fills[L::kGroups];
    const int gi = threadIdx.x / L::G;
    const int64_t r = (int64_t)blockIdx.x * L::kGroups + gi;
    if (r >= a.n_rows)
        return;
    Group<L::G> g(threadIdx.x % L::G, &scratch);
    const int cap = min(a.k, a.n);
    uint64_t *list = lists + (int64_t)gi * cap;
    uint32_t *fill = fills + gi;
    if (g.t == 0)
        *fill = 0;
    const char *src = a.logits + r * a.stride;
    const Row<TYPE, L::G, L::NV, L::VEC, L::RESIDENT> row(src, a.n, g.t);

    const float c = a.inv_t * kLog2e;
    Softmax sm = {-__builtin_inff(), 0.0f};
    Cmp top = E::lowest();
    uint32_t valid = 0;
    row.each([&](int, int32_t, const Piece<TYPE, L::VEC> &p) {
        float z[L::VEC], zm = -__builtin_inff();
#pragma unroll
        for (int u = 0; u < L::VEC; ++u) {
            const Cmp v = p.get(u);
            const bool in = v > E::lowest();
            valid += in;
            top = in && v > top ? v : top;
            z[u] = in ? E::to_float(v) : -__builtin_inff();
            zm = fmaxf(zm, z[u]);
        }
        sm.raise(zm, c);
        const float from = sm.from();
#pragma unroll
        for (int u = 0; u < L::VEC; ++u)
            sm.s += __builtin_amdgcn_exp2f((z[u] - from) * c);
    });
    if (a.log_norm) {
        sm = combine(g, sm, c);
        if (g.t == 0)
            a.log_norm[r] = sm.log_norm(a.inv_t);
    }
    const uint32_t k = min((uint32_t)a.k, g.reduce(valid, Add()));
    top = g.reduce(top, Max());

    uint32_t lo = E::kFirstKey, hi = E::key(top) + 1;     // count(>= lo) >= k > count(>= hi)
    while (k && hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const Cmp at = E::from_key(mid);
        uint32_t count = 0;
        row.each([&](int, int32_t, const Piece<TYPE, L::VEC> &p) {
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                count += p.get(u) >= at;
        });
        if (g.reduce(count, Add()) >= k)
            lo = mid;
        else
            hi = mid;
    }
    const Cmp tau = E::from_key(lo);
    g.barrier();
    if (k)
        row.each([&](int, int32_t i, const Piece<TYPE, L::VEC> &p) {
#pragma unroll
            for (int u = 0; u < L::VEC; ++u) {
                const Cmp v = p.get(u);
                if (v > tau)
                    list[atomicAdd(fill, 1u)] = (uint64_t)E::key(v) << 32 | ~(uint32_t)(i + u);
            }
        });
    g.barrier();
    uint32_t taken = *fill;                               // then the equal ones, by class
    g.barrier();
    row.each([&](int, int32_t i, const Piece<TYPE, L::VEC> &p) {
        if (taken >= k)
            return;
        uint32_t mine = 0, total;
#pragma unroll
        for (int u = 0; u < L::VEC; ++u)
            mine += p.get(u) == tau;
        uint32_t place = taken + g.scan(mine, total);
        taken += total;
#pragma unroll
        for (int u = 0; u < L::VEC; ++u)
            if (p.get(u) == tau) {
                if (place < k)
                    list[place] = (uint64_t)lo << 32 | ~(uint32_t)(i + u);
                ++place;
            }
    });
    g.barrier();

    char *values = a.values + r * a.k * E::kBytes;
    int32_t *indices = a.indices + r * a.k;
    for (uint32_t e = g.t; e < (uint32_t)a.k; e += L::G) {
        uint32_t to = e;
        int32_t cls = -1;
        if (e < k) {
            const uint64_t mine = list[e];
            to = 0;
            for (uint32_t f = 0; f < k; ++f)
                to += list[f] > mine;
            cls = (int32_t)~(uint32_t)mine;
        }
        indices[to] = cls;
        if constexpr (E::kBytes == 4)
            reinterpret_cast<uint32_t *>(values)[to] =
                cls >= 0 ? reinterpret_cast<const uint32_t *>(src)[cls]
                         : TYPE == kI32 ? 0x80000000u : 0xFF800000u;
        else
            reinterpret_cast<uint16_t *>(values)[to] =
                cls >= 0 ? reinterpret_cast<const uint16_t *>(src)[cls]
                         : TYPE == kF16 ? 0xFC00u : 0xFF80u;
    }
}

}  // namespace

hipError_t launch_top_logits(const void *logits, int32_t type, int64_t n_rows, int32_t n,
                             int64_t row_stride, int32_t k, float inv_t, void *values,
                             int32_t *indices, float *log_norm, hipStream_t stream)
{
    return with_type(type, [&](auto ty) {
        constexpr int TYPE = decltype(ty)::value;
        const TopArgs a = {static_cast<const char *>(logits), row_stride * Elem<TYPE>::kBytes,
                           n_rows, n, k, inv_t, static_cast<char *>(values), indices, log_norm};
        return with_layout<TYPE>(n, 0, [&](auto layout) {
            typedef decltype(layout) L;
            const size_t lds = (size_t)L::kGroups * (k < n ? k : n) * sizeof(uint64_t);
            k_top<TYPE, L><<<(uint32_t)((n_rows + L::kGroups - 1) / L::kGroups), L::kBlock, lds,
                             stream>>>(a);
            return hipGetLastError();
        });
    });
}

}  // namespace bl
