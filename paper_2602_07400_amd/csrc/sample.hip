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
// first classes of (key == tau).  For a top-p, sums of w in 2048 intervals of x, in
// fixed point so that their order does not matter, say which interval the prefix ends
// in, and that one's classes are put in order; where neither list holds them, tau comes
// from bisection on the key: on counts for top-k, on sums of w for top-p.
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

// Lanes of each wave whose largest logits bound the list of a top-p without a top-k.
constexpr uint32_t kNucleusLanes = 4;
// Intervals of x for the sums of w: kBins of them down to -kRange, where w is 4e-11.
constexpr float kRange = 24.0f;
constexpr float kFixed = 1099511627776.0f;                // 2^40 a unit of w

template <int TYPE, class L>
__global__ __launch_bounds__(L::kBlock, L::kWavesPerSimd) void k_sample(SampleArgs a)
{
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    typedef Piece<TYPE, L::VEC> P;
    constexpr int G = L::G;
    constexpr bool kLists = G >= kWave;
    constexpr int kCounted = kLists ? L::kCounted : 1;
    constexpr int kSlots = !kLists ? 1 : G > kWave && L::kList < (int)kBins ? (int)kBins : L::kList;
    __shared__ Scratch scratch;
    __shared__ uint64_t lists[kLists ? L::kGroups : 1][kSlots];
    __shared__ uint64_t placed[kLists ? L::kGroups : 1][kCounted];
    __shared__ float numbers[kLists ? L::kGroups : 1][kCounted];
    __shared__ uint32_t fills[L::kGroups];
    const int gi = threadIdx.x / G;
    const int64_t r = (int64_t)blockIdx.x * L::kGroups + gi;
    if (r >= a.n_rows)
        return;
    Group<G> g(threadIdx.x % G, &scratch);
    const char *src = a.logits + r * a.stride;
    const float *noise = a.noise + r * a.noise_stride;
    Row<TYPE, G, L::NV, L::VEC, L::RESIDENT> row(src, a.n, g.t);
    const float temperature = a.temperatures ? a.temperatures[r] : a.temperature;
    const float top_p = a.top_ps ? a.top_ps[r] : a.top_p;
    const float min_p = a.min_ps ? a.min_ps[r] : a.min_p;
    int32_t top_k = a.top_ks ? a.top_ks[r] : a.top_k;
    if (top_k <= 0 || top_k > a.n)
        top_k = a.n;
    const bool by_k = top_k < a.n, by_p = top_p < 1.0f;
    const float inv_t = 1.0f / temperature;

    // the lane's and its pieces' largest logits and, for a top-p of all classes, the
    // softmax's sum, as the row arrives
    Cmp mine = E::lowest(), most[L::NV];
    Softmax sm = {-__builtin_inff(), 0.0f};
    const bool of_all = by_p && !by_k && temperature > 0.0f;
    const float c = inv_t * kLog2e;
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
        if (of_all) {
            sm.raise(vm > E::lowest() ? E::to_float(vm) : -__builtin_inff(), c);
            const float from = sm.from();
#pragma unroll
            for (int u = 0; u < L::VEC; ++u) {
                const Cmp v = p.get(u);
                sm.s += v > E::lowest() ? __builtin_amdgcn_exp2f((E::to_float(v) - from) * c)
                                        : 0.0f;
            }
        }
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
    float row_mass = 0.0f;                                // sum of w
    if (of_all) {
        if (ftop < __builtin_inff())
            sm.raise(ftop, c);
        else
            sm.s = 0.0f;                                  // w = 1 at +inf, else 0
        if (ftop == __builtin_inff())
            row.each([&](int, int32_t, const P &p) {
#pragma unroll
                for (int u = 0; u < L::VEC; ++u)
                    sm.s += p.get(u) == top ? 1.0f : 0.0f;
            });
        row_mass = g.reduce(sm.s, Add());
    }
    float sum = 0.0f;                                     // of the kept w
    float best = -__builtin_inff(), best_x = 0.0f;        // x + g of the lane's best class
    int32_t best_class = 0;
    const auto finish = [&](auto first) __attribute__((always_inline)) {
        const uint64_t own = best > -__builtin_inff()
                                 ? entry(Elem<kF32>::key(best), best_class) : 0;
        const uint64_t won = g.reduce(own, Max());
        sum = g.reduce(sum, Add());
        int32_t token = best_class;
        if (!won) {
            token = first();
            best_x = 0.0f;
        }
        if (won ? own == won : g.t == 0) {
            a.token[r] = token;
            if (a.log_prob)
                a.log_prob[r] = best_x - logf(sum);
        }
    };

    const Cmp all = E::from_key(E::kFirstKey);
    uint32_t *fill = &fills[gi];
    if constexpr (kLists) {
        constexpr uint32_t W = G / kWave;
        uint64_t *list = lists[gi];
        uint32_t lo = E::kFirstKey;
        const uint32_t lanes = by_k ? (top_k + W - 1) / W : kNucleusLanes;
        if ((by_k || by_p) && lanes <= kWave)
            lo = max(lo, ~g.reduce(~wave_mth(mine > E::lowest() ? E::key(mine) : 0, lanes),
                                   Max()));
        for (int attempt = 0; (by_k || by_p) && attempt < 2; ++attempt) {
            const uint32_t found = collect<TYPE, L>(g, row, most, E::from_key(lo), false, top,
                                                    list, fill);
            if (found > (uint32_t)L::kList) {
                if (!by_k || top_k > L::kList || attempt)
                    break;
                if constexpr (G > kWave)
                    lo = raise_bound<TYPE, L>(g, row, lo, E::key(top), top_k, (uint32_t *)list);
                continue;
            }
            const bool counted = found <= (uint32_t)kCounted;
            uint64_t *sorted = counted ? placed[gi] : list;
            if (counted)
                place_entries(g, list, found, sorted, numbers[gi],
                              [&](uint64_t x) { return noise[class_of(x)]; });
            else
                sort_entries(g, list, found);
            const uint32_t n = by_k ? min(found, (uint32_t)top_k) : found;
            // sums of w before each entry: a run of entries a lane
            const uint32_t run = (n + G - 1) / G, e0 = min(n, g.t * run), e1 = min(n, e0 + run);
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
                        const float score = x + (counted ? numbers[gi][e] : noise[cls]);
                        if (score > best || (score == best && cls < best_class)) {
                            best = score;
                            best_x = x;
                            best_class = cls;
                        }
                    }
                    before += we;
                }
                finish([&] { return class_of(sorted[0]); });
                return;
            }
            if (G > kWave)
                break;
            lo = E::kFirstKey;                            // a wave's list holds the row
        }
    }

    const auto mass_from = [&](Cmp at) __attribute__((always_inline)) {
        float part = 0.0f;                                // sum of w over logits >= at
        row.each([&](int j, int32_t, const P &p) {
            if constexpr (L::RESIDENT)
                if (!(most[j] >= at))
                    return;
#pragma unroll
            for (int u = 0; u < L::VEC; ++u) {
                const Cmp v = p.get(u);
                part += v >= at ? exp_fast(x_of(v)) : 0.0f;
            }
        });
        return g.reduce(part, Add());
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
    // the kept prefix: keys above tau, and of those equal to it `ties`, or the classes
    // up to `last`
    const uint32_t end = E::key(top) + 1;
    uint32_t tau = E::kFirstKey, ties = 0xFFFFFFFFu;
    int32_t last = INT32_MAX;
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
                const float more = tau + 1 == end ? 0.0f : mass_from(E::from_key(tau + 1));
                target = more + (float)ties * exp_fast(x_of(E::from_key(tau)));
            } else {
                target = mass_from(all);
            }
        }
        target *= top_p;
        uint32_t lo = tau, hi = end;                      // mass(>= lo) >= target > mass(>= hi)
        float above = 0.0f;                               // mass(>= hi)
        bool found_last = false;
        if constexpr (G > kWave)
            if (!by_k) {
                constexpr uint32_t kRun = kBins / G;
                unsigned long long *bins = reinterpret_cast<unsigned long long *>(lists[gi]);
                const float scale = (float)kBins / kRange;
                const auto bin_of = [&](Cmp v) __attribute__((always_inline)) {
                    return -x_of(v) * scale;              // grows as v falls; may be inf
                };
                g.barrier();
                for (uint32_t b = g.t; b < kBins; b += G)
                    bins[b] = 0;
                g.barrier();
                row.each([&](int, int32_t, const P &p) {
#pragma unroll
                    for (int u = 0; u < L::VEC; ++u) {
                        const Cmp v = p.get(u);
                        const float b = bin_of(v);
                        if (v >= all && b < (float)kBins)
                            atomicAdd(&bins[(uint32_t)b],
                                      (unsigned long long)(exp_fast(x_of(v)) * kFixed));
                    }
                });
                g.barrier();
                const unsigned long long goal = (unsigned long long)(target * kFixed);
                unsigned long long part = 0, total;
                for (uint32_t b = 0; b < kRun; ++b)
                    part += bins[g.t * kRun + b];
                unsigned long long before = g.scan(part, total), base = 0;
                uint32_t in = 0;                          // 1 + the bin that reaches it
                for (uint32_t b = 0; b < kRun; ++b) {
                    const unsigned long long here = bins[g.t * kRun + b];
                    if (before < goal && before + here >= goal) {
                        in = g.t * kRun + b + 1;
                        base = before;
                    }
                    before += here;
                }
                in = g.reduce(in, Max());
                base = g.reduce((uint64_t)base, Max());
                if (in) {
                    // its keys: [lo, hi)
                    const auto first_key = [&](float bound) __attribute__((always_inline)) {
                        uint32_t no = E::kFirstKey - 1, yes = end - 1;
                        while (yes - no > 1) {
                            const uint32_t mid = no + (yes - no) / 2;
                            if (bin_of(E::from_key(mid)) < bound)
                                yes = mid;
                            else
                                no = mid;
                        }
                        return yes;
                    };
                    lo = first_key((float)in);
                    hi = in == 1 ? end : first_key((float)(in - 1));
                    above = (float)base / kFixed;
                    const Cmp to = E::from_key(in == 1 ? lo : hi);
                    uint64_t *list = lists[gi];
                    const uint32_t found = collect<TYPE, L>(g, row, most, E::from_key(lo),
                                                            in != 1, to, list, fill);
                    if (found && found <= (uint32_t)L::kList) {
                        sort_entries(g, list, found);
                        const uint32_t run = (found + G - 1) / G, e0 = min(found, g.t * run),
                                       e1 = min(found, e0 + run);
                        float w = 0.0f, listed;
                        for (uint32_t e = e0; e < e1; ++e)
                            w += exp_fast(x_of(E::from_key(key_of(list[e]))));
                        float sums = above + g.scan(w, listed);
                        uint32_t kept = 1;
                        for (uint32_t e = e0; e < e1; ++e) {
                            if (sums < target)
                                kept = e + 1;
                            sums += exp_fast(x_of(E::from_key(key_of(list[e]))));
                        }
                        const uint64_t x = list[g.reduce(kept, Max()) - 1];
                        tau = key_of(x);
                        last = class_of(x);
                        found_last = true;
                    }
                }
            }
        if (!found_last) {
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
            const uint32_t take = need >= 4.0e9f ? 0xFFFFFFFFu
                                                 : need > 1.0f ? (uint32_t)need : 1u;
            ties = lo == tau ? min(take, ties) : take;
            tau = lo;
        }
    }
    const Cmp at = E::from_key(tau);
    if (ties != 0xFFFFFFFFu) {                            // the last kept class equal to tau
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
        float number[L::VEC];
        if (i + L::VEC <= a.n) {
            __builtin_memcpy(number, noise + i, sizeof number);
        } else {
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                number[u] = i + u < a.n ? noise[i + u] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < L::VEC; ++u) {
            const Cmp v = p.get(u);
            const float x = x_of(v);
            const bool kept = (v > at || (v == at && i + u <= last)) && (x >= floor_x || v == top);
            sum += kept ? exp_fast(x) : 0.0f;
            const float score = x + number[u];
            if (kept && score > best) {                   // (the lane's classes ascend)
                best = score;
                best_x = x;
                best_class = i + u;
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
