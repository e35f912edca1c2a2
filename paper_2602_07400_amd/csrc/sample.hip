// A class per row, drawn from its logits under temperature, top-k, top-p and min-p
// with given random numbers.
//
// With x_i = (l_i - max l) * (1 / T), w_i = e^x_i and the row's order (descending
// logit, ascending class):
//   top-k   keeps the first k classes of the order;
//   top-p   of those, the shortest prefix whose sum of w reaches p times their sum;
//   min-p   of those, the ones with x_i >= log(min_p).
// The draw is the kept class with the largest x_i + g_i, g_i given standard Gumbel
// numbers: P(class) = w_i / sum of the kept w.  (One number a class makes the winner
// a comparison of elementary sums; one uniform number a row would make it depend on
// the rounding of a prefix sum over all classes.)
//
// Every filter keeps a prefix of the order.  Where it is short, its classes are among
// those of a list in LDS, found from the lanes' largest logits as in top_logits.hip
// and put in order: top-k is a place, top-p a prefix sum, and the kept classes' numbers
// are all that is read of the noise.  Otherwise the kept set is (key > tau) and the
// first classes of (key == tau), tau from bisection on the key: on counts for top-k,
// on sums of w for top-p.
#include "logit_rows.h"

namespace bl {
namespace {

using namespace rows;

struct SampleArgs {
    const char *logits;
    int64_t stride;                     // bytes from row to row
    int64_t n_rows;
    int32_t n;
    const float *noise;                 // [rows][n]
    int64_t noise_stride;               // elements from row to row
    float temperature, top_p, min_p;    // where the arrays below are NULL
    int32_t top_k;
    const float *temperatures, *top_ps, *min_ps;
    const int32_t *top_ks;
    int32_t *token;                     // [rows]
    float *log_prob;                    // [rows] or NULL
};

// Places up to here come from counting the larger entries, more from a sort.
constexpr uint32_t kCounted = 128;
// Lanes of each wave whose largest logits bound the list of a top-p without a top-k.
constexpr uint32_t kNucleusLanes = 16;

template <int TYPE, class L>
__global__ __launch_bounds__(L::kBlock) void k_sample(SampleArgs a)
{
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    typedef Piece<TYPE, L::VEC> P;
    constexpr int G = L::G;
    constexpr bool kLists = G >= kWave;
    __shared__ Scratch scratch;
    __shared__ uint64_t lists[kLists ? L::kGroups : 1][kLists ? L::kList : 1];
    __shared__ uint64_t placed[kLists ? L::kGroups : 1][kCounted];
    __shared__ uint32_t fills[L::kGroups];
    const int gi = threadIdx.x / G;
    const int64_t r = (int64_t)blockIdx.x * L::kGroups + gi;
    if (r >= a.n_rows)
        return;
    Group<G> g(threadIdx.x % G, &scratch);
    if (g.t == 0)
        fills[gi] = 0;
    const char *src = a.logits + r * a.stride;
    const float *noise = a.noise + r * a.noise_stride;
    Row<TYPE, G, L::NV, L::VEC, L::RESIDENT> row(src, a.n, g.t);
    const float temperature = a.temperatures ? a.temperatures[r] : a.temperature;
    const float top_p = a.top_ps ? a.top_ps[r] : a.top_p;
    const float min_p = a.min_ps ? a.min_ps[r] : a.min_p;
    int32_t top_k = a.top_ks ? a.top_ks[r] : a.top_k;
    if (top_k <= 0 || top_k > a.n)
        top_k = a.n;
    const float inv_t = 1.0f / temperature;

    // the lane's and its pieces' largest logits
    Cmp mine = E::lowest(), most[L::NV];
    row.each([&](int j, int32_t, const P &p) {
        Cmp vm = E::lowest();
#pragma unroll
        for (int u = 0; u < L::VEC; ++u) {
            const Cmp v = p.get(u);
            vm = v > vm ? v : vm;
        }
        mine = vm > mine ? vm : mine;
        if constexpr (L::RESIDENT)
            most[j] = vm;
    });
    const Cmp top = g.reduce(mine, Max());
    const auto first_class = [&]() __attribute__((always_inline)) {
        uint32_t first = 0;                               // of the largest, ~class
        if (mine == top)
            row.each([&](int, int32_t i, const P &p) {
#pragma unroll
                for (int u = 0; u < L::VEC; ++u)
                    if (p.get(u) == top)
                        first = max(first, ~(uint32_t)(i + u));
            });
        return (int32_t)~g.reduce(first, Max());
    };
    if (!(top > E::lowest()) || !(temperature > 0.0f)) {
        const bool any = top > E::lowest();               // greedy, or nothing to draw from
        const int32_t token = any ? first_class() : -1;
        if (g.t == 0) {
            a.token[r] = token;
            if (a.log_prob)
                a.log_prob[r] = any ? 0.0f : -__builtin_inff();
        }
        return;
    }

    const float ftop = E::to_float(top);
    const float floor_x = min_p > 0.0f ? logf(min_p) : -__builtin_inff();
    const auto x_of = [&](Cmp v) __attribute__((always_inline)) {
        return v == top ? 0.0f : (E::to_float(v) - ftop) * inv_t;
    };
    const auto mass_from = [&](Cmp at) __attribute__((always_inline)) {
        float sum = 0.0f;                                 // of w over logits >= at
        row.each([&](int j, int32_t, const P &p) {
            if constexpr (L::RESIDENT)
                if (!(most[j] >= at))
                    return;
#pragma unroll
            for (int u = 0; u < L::VEC; ++u) {
                const Cmp v = p.get(u);
                sum += v >= at ? exp_fast(x_of(v)) : 0.0f;
            }
        });
        return g.reduce(sum, Add());
    };
    const auto count_from = [&](Cmp at) __attribute__((always_inline)) {
        uint32_t count = 0;
        row.each([&](int j, int32_t, const P &p) {
            if constexpr (L::RESIDENT)
                if (!(most[j] >= at))
                    return;
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                count += p.get(u) >= at;
        });
        return g.reduce(count, Add());
    };
    float sum = 0.0f;                                     // of the kept w
    uint64_t best = 0;                                    // (key of x + g, ~class)
    const auto draw = [&](float x, int32_t cls, float number) __attribute__((always_inline)) {
        const float score = x + number;
        if (score > -__builtin_inff()) {
            const uint64_t s = entry(Elem<kF32>::key(score), cls);
            best = s > best ? s : best;
        }
    };
    const auto finish = [&](auto first) __attribute__((always_inline)) {
        best = g.reduce(best, Max());
        sum = g.reduce(sum, Add());
        const int32_t token = best ? class_of(best) : first();
        if (g.t == 0) {
            a.token[r] = token;
            if (a.log_prob)
                a.log_prob[r] = x_of(load_one<TYPE>(src, token)) - logf(sum);
        }
    };

    const bool by_k = top_k < a.n, by_p = top_p < 1.0f;
    const Cmp all = E::from_key(E::kFirstKey);
    float row_mass = 0.0f;
    if (by_p && !by_k)
        row_mass = mass_from(all);

    if constexpr (kLists) {
        constexpr uint32_t W = G / kWave;
        const uint32_t lanes = by_k ? (top_k + W - 1) / W : kNucleusLanes;
        if ((by_k || by_p) && lanes <= kWave) {
            uint64_t *list = lists[gi], *sorted = placed[gi];
            uint32_t *fill = &fills[gi];
            const uint32_t key = mine > E::lowest() ? E::key(mine) : 0;
            const uint32_t lo = max((uint32_t)E::kFirstKey,
                                    ~g.reduce(~wave_mth(key, lanes), Max()));
            const Cmp at = E::from_key(lo);
            row.each([&](int j, int32_t i, const P &p) {
                if constexpr (L::RESIDENT)
                    if (!(most[j] >= at))
                        return;
#pragma unroll
                for (int u = 0; u < L::VEC; ++u) {
                    const Cmp v = p.get(u);
                    if (v >= at) {
                        const uint32_t to = atomicAdd(fill, 1u);
                        if (to < (uint32_t)L::kList)
                            list[to] = entry(E::key(v), i + u);
                    }
                }
            });
            g.barrier();
            const uint32_t found = *fill;
            if (found <= (uint32_t)L::kList) {
                if (found <= kCounted) {
                    for (uint32_t e = g.t; e < found; e += G) {
                        const uint64_t x = list[e];
                        sorted[place_of(x, list, found)] = x;
                    }
                    g.barrier();
                } else {
                    sort_entries(g, list, found);
                    sorted = list;
                }
                const uint32_t n = by_k ? min(found, (uint32_t)top_k) : found;
                // sums of w before each entry: a run of entries a lane
                const uint32_t run = (n + G - 1) / G, e0 = min(n, g.t * run),
                               e1 = min(n, e0 + run);
                float w = 0.0f, total;
                for (uint32_t e = e0; e < e1; ++e)
                    w += exp_fast(x_of(E::from_key(key_of(sorted[e]))));
                float before = g.scan(w, total);
                const float target = top_p * (by_k ? total : row_mass);
                // the list reaches the target, or holds every class
                if (!by_p || by_k || total >= target || lo == E::kFirstKey) {
                    for (uint32_t e = e0; e < e1; ++e) {
                        const float x = x_of(E::from_key(key_of(sorted[e])));
                        const float we = exp_fast(x);
                        if (e == 0 || ((!by_p || before < target) && x >= floor_x)) {
                            const int32_t cls = class_of(sorted[e]);
                            sum += we;
                            draw(x, cls, noise[cls]);
                        }
                        before += we;
                    }
                    finish([&] { return class_of(sorted[0]); });
                    return;
                }
            }
        }
    }

    // the kept prefix: keys above tau, and `ties` of those equal to it
    const uint32_t end = E::key(top) + 1;
    uint32_t tau = E::kFirstKey, ties = 0xFFFFFFFFu;
    if (by_k && count_from(all) > (uint32_t)top_k) {
        uint32_t hi = end;                                // count(>= tau) >= k > count(>= hi)
        while (hi - tau > 1) {
            const uint32_t mid = tau + (hi - tau) / 2;
            if (count_from(E::from_key(mid)) >= (uint32_t)top_k)
                tau = mid;
            else
                hi = mid;
        }
        ties = top_k - (hi == end ? 0 : count_from(E::from_key(hi)));
    }
    if (by_p) {
        float target = row_mass;
        if (by_k) {
            if (ties != 0xFFFFFFFFu) {
                const float above = tau + 1 == end ? 0.0f : mass_from(E::from_key(tau + 1));
                target = above + (float)ties * exp_fast(x_of(E::from_key(tau)));
            } else {
                target = mass_from(all);
            }
        }
        target *= top_p;
        uint32_t lo = tau, hi = end;                      // mass(>= lo) >= target > mass(>= hi)
        float above = 0.0f;                               // mass(>= hi)
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            const float mass = mass_from(E::from_key(mid));
            if (mass >= target) {
                lo = mid;
            } else {
                hi = mid;
                above = mass;
            }
        }
        // equal classes until the target: at least one
        const float w = exp_fast(x_of(E::from_key(lo)));
        const float need = ceilf((target - above) / w);
        const uint32_t take = need >= 4.0e9f ? 0xFFFFFFFFu : need > 1.0f ? (uint32_t)need : 1u;
        ties = lo == tau ? min(take, ties) : take;
        tau = lo;
    }
    const Cmp at = E::from_key(tau);
    // the last kept class equal to tau
    int32_t last = INT32_MAX;
    if (ties != 0xFFFFFFFFu) {
        uint32_t seen = 0;
        int32_t equal = -1;
        row.each([&](int, int32_t i, const P &p) {
            if (seen >= ties)
                return;
            uint32_t here = 0, total;
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                here += p.get(u) == at;
            uint32_t place = seen + g.scan(here, total);
            seen += total;
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                if (p.get(u) == at && place++ < ties)
                    equal = i + u;
        });
        last = g.reduce(equal, Max());
    }
    row.each([&](int j, int32_t i, const P &p) {
        if constexpr (L::RESIDENT)
            if (!(most[j] >= at))
                return;
#pragma unroll
        for (int u = 0; u < L::VEC; ++u) {
            const Cmp v = p.get(u);
            const float x = x_of(v);
            if ((v > at || (v == at && i + u <= last)) && (x >= floor_x || v == top)) {
                sum += exp_fast(x);
                draw(x, i + u, noise[i + u]);
            }
        }
    });
    finish(first_class);
}

}  // namespace

hipError_t launch_sample(const void *logits, int32_t type, int64_t n_rows, int32_t n,
                         int64_t row_stride, const float *noise, int64_t noise_stride,
                         const SampleParams &sp, int32_t *token, float *log_prob,
                         hipStream_t stream)
{
    return with_type(type, [&](auto ty) {
        constexpr int TYPE = decltype(ty)::value;
        const SampleArgs a = {static_cast<const char *>(logits),
                              row_stride * Elem<TYPE>::kBytes, n_rows, n, noise, noise_stride,
                              sp.temperature, sp.top_p, sp.min_p, sp.top_k, sp.temperatures,
                              sp.top_ps, sp.min_ps, sp.top_ks, token, log_prob};
        return with_layout<TYPE>(n, 0, [&](auto layout) {
            typedef decltype(layout) L;
            k_sample<TYPE, L><<<(uint32_t)((n_rows + L::kGroups - 1) / L::kGroups), L::kBlock, 0,
                                stream>>>(a);
            return hipGetLastError();
        });
    });
}

}  // namespace bl
