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
// first classes of (key == tau); tau is narrowed down by counts, for a top-k, or sums
// of w, for a top-p, in ever narrower intervals.  Rows of a part of a wave find it by
// bisection.
//
// What bounds it: short prefixes, the block's chain after the load (1 x 131072 bf16, top-k
// 50 and top-p 0.95: 15 us, of which 4 to 5 are the load); wide ones, the passes over
// the row, of 25 instructions and a 64-bit LDS atomic an element each: 256 x 131072 with
// parameters per row 92 us, when a few rows keep thousands of classes, the others are done
// in 20 and the VALU is active in 12 of 100 cycles; without filters, HBM and the turns of
// loading and drawing that a row held for its maximum takes: 1024 x 50021 float32 87 us,
// 4.7 TB/s, the VALU active in 42 of 100 cycles.
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

    void skip(int64_t rows)
    {
        const auto on = [](auto *&p, int64_t by) { p = p ? p + by : p; };
        logits += rows * stride;
        on(noise, rows * noise_stride);
        on(temperatures, rows);
        on(top_ps, rows);
        on(min_ps, rows);
        on(top_ks, rows);
        token += rows;
        on(log_prob, rows);
    }
};

// Lanes whose largest logits bound the list of a top-p without a top-k.
constexpr uint32_t kNucleusLanes = 64;

// PLAIN: no filter in any row, so that every class and number counts: the row stays in
// registers for the draw, and the first numbers are loaded behind it.  Otherwise rows
// without a filter are read twice.
template <int TYPE, class L, bool PLAIN>
__global__ __launch_bounds__(L::kBlock, PLAIN ? L::kWavesPerSimd : 4) void k_sample(SampleArgs a)
{
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    typedef Piece<TYPE, L::VEC> P;
    constexpr int G = L::G;
    constexpr bool kLists = G >= kWave && !PLAIN;
    constexpr int kCounted = kLists ? L::kCounted : 1;
    __shared__ Scratch scratch;
    __shared__ uint64_t lists[kLists ? L::kGroups : 1][kLists ? L::kList : 1];
    __shared__ uint64_t placed[kLists ? L::kGroups : 1][kCounted];
    __shared__ float numbers[kLists ? L::kGroups : 1][kCounted];
    __shared__ uint32_t fills[L::kGroups];
    const int gi = group_of<G>();
    const int64_t r = (int64_t)blockIdx.x * L::kGroups + gi;
    if (r >= a.n_rows)
        return;
    Group<G> g(threadIdx.x - gi * G, &scratch);
    const char *src = a.logits + r * a.stride;
    const float *noise = a.noise + r * a.noise_stride;
    // (only what plain draws and bisection read again stays in registers)
    Row<TYPE, G, L::NV, L::VEC, L::RESIDENT, (PLAIN || G < kWave)> row(src, a.n, g.t);
    const float temperature = a.temperatures ? a.temperatures[r] : a.temperature;
    const float top_p = PLAIN ? 1.0f : a.top_ps ? a.top_ps[r] : a.top_p;
    const float min_p = PLAIN ? 0.0f : a.min_ps ? a.min_ps[r] : a.min_p;
    int32_t top_k = PLAIN ? a.n : a.top_ks ? a.top_ks[r] : a.top_k;
    if (top_k <= 0 || top_k > a.n)
        top_k = a.n;
    const bool by_k = top_k < a.n, by_p = top_p < 1.0f;
    const float inv_t = inverse(temperature);

    constexpr int kRoom = TYPE == kF16 && L::NV == 16 ? 16 : 32;   // registers for them
    constexpr int kAhead = !L::RESIDENT ? 1 : L::NV < kRoom / L::VEC ? L::NV : kRoom / L::VEC;
    static_assert(!L::RESIDENT || L::NV % kAhead == 0, "whole batches");
    typedef float Numbers[kAhead][L::VEC];
    const auto numbers_of = [&](int32_t i, float (&to)[L::VEC]) __attribute__((always_inline)) {
        const float *from = noise + i + (uint32_t)(g.t * L::VEC);   // i: of the group's first
        if (i + L::kSpan <= a.n) {
            __builtin_memcpy(to, from, sizeof to);
        } else {
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                to[u] = 0.0f;
            for (int u = min(a.n - i - g.t * L::VEC, L::VEC) - 1; u >= 0; --u) {
#pragma unroll
                for (int k = L::VEC - 1; k > 0; --k)
                    to[k] = to[k - 1];
                to[0] = from[u];
            }
        }
    };
    const bool unfiltered = !by_k && !by_p && !(min_p > 0.0f) && temperature > 0.0f;
    Numbers early;
    if constexpr (L::RESIDENT && PLAIN)
        if (unfiltered)
            static_for<kAhead>([&](auto j) __attribute__((always_inline)) {
                numbers_of(j * L::kSpan, early[j]);
            });

    // the lane's and its pieces' largest logits and, for a top-p of all classes, the
    // softmax's sum, as the row arrives
    Cmp mine = E::lowest(), most[L::NV];
    static_for<L::NV>([&](auto j) __attribute__((always_inline)) { most[j] = E::lowest(); });
    Softmax<TYPE, !L::RESIDENT> sm;
    const bool of_all = by_p && !by_k && temperature > 0.0f && kLists;
    const float c = inv_t * kLog2e;
    row.each([&](auto j, int32_t, const P &p) {
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
            sm.raise(vm, c);
            const Cmp from = sm.from();
            float part = sm.start();
#pragma unroll
            for (int u = 0; u < L::VEC; ++u) {
                const Cmp v = p.get(u);
                part += v > E::lowest() ? __builtin_amdgcn_exp2f(E::minus(v, from) * c) : 0.0f;
            }
            sm.add(part);
        }
    });
    const Cmp top = g.reduce(mine, Max());
    const auto first_class = [&]() __attribute__((always_inline)) {
        uint32_t first = 0;                               // of the largest, ~class
        const auto search = [&](int32_t i, const P &p) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                if (p.get(u) == top)
                    first = max(first, ~(uint32_t)(i + u));
        };
        if constexpr (L::RESIDENT) {
            const uint32_t hits = pieces_from<L>(most, top);
            if (hits) {                                   // the lane's first piece with it
                const int32_t i = (__builtin_ctz(hits) * G + g.t) * L::VEC;
                P p;
                p.load(src, 0, i, a.n);
                search(i, p);
            }
        } else {
            row.stream(search);
        }
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

    // (a row with +inf draws among those: x = 0 there, the minimum's answer to the NaN of
    // inf - inf, and -inf elsewhere)
    const bool endless = E::to_float(top) == __builtin_inff();
    const float floor_x = min_p > 0.0f ? logf(min_p) : -__builtin_inff();
    const auto x_of = [&](Cmp v) __attribute__((always_inline)) {
        return fminf(E::minus(v, top) * inv_t, 0.0f);
    };
    float row_mass = 0.0f;                                // sum of w
    if (of_all) {
        if (endless) {
            sm.s = 0.0f;
            row.stream([&](int32_t, const P &p) {
#pragma unroll
                for (int u = 0; u < L::VEC; ++u)
                    sm.s += p.get(u) == top ? 1.0f : 0.0f;
            });
        } else {
            sm.raise(top, c);
        }
        row_mass = g.reduce(sm.s, Add());
    }
    Total<!L::RESIDENT> sum;                              // of the kept w
    float best = -__builtin_inff(), best_x = 0.0f;        // the lane's best x + g (and x),
    int32_t best_class = 0;                               // and its class
    const auto finish = [&](auto &h, auto first, auto x_best) __attribute__((always_inline)) {
        const uint64_t own = best > -__builtin_inff()
                                 ? entry(Elem<kF32>::key(best), best_class) : 0;
        const uint64_t won = h.reduce(own, Max());
        const float total = h.reduce(sum.s, Add());
        const int32_t token = won ? best_class : first();
        if (won ? own == won : g.t == 0) {
            a.token[r] = token;
            if (a.log_prob)
                a.log_prob[r] = (won ? x_best() : 0.0f) - logf(total);
        }
    };
    const auto x_listed = [&] { return best_x; };
    const auto x_loaded = [&] { return x_of(load_one<TYPE>(src, best_class)); };

    // a draw among a piece's logits above `in`, if the piece's classes end at or before
    // `last`, and above `out` in classes after it
    const auto draw = [&](Cmp in, Cmp out, int32_t last, int32_t i, const P &p,
                          const float (&number)[L::VEC]) __attribute__((always_inline)) {
        const bool split = i <= last && i + L::VEC - 1 > last;
        const Cmp over = i <= last ? in : out;
        int at = -1;
        float part = sum.start();
        const auto one = [&](int u, bool kept) __attribute__((always_inline)) {
            const float x = x_of(p.get(u));
            part += kept ? exp_fast(x) : 0.0f;
            const float score = kept ? x + number[u] : -__builtin_inff();
            at = score > best ? u : at;                   // (the lane's classes ascend)
            best = fmaxf(best, score);
        };
        if (!__any(split)) {
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                one(u, p.get(u) > over);
        } else {
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                one(u, p.get(u) > (i + u <= last ? in : out));
        }
        sum.add(part);
        best_class = at >= 0 ? i + at : best_class;
    };
    const auto draw_streamed = [&](Cmp at, Cmp in, int32_t last) __attribute__((always_inline)) {
        uint32_t hits = pieces_from<L>(most, at);
        constexpr int kFlight = L::RESIDENT && L::NV < 4 ? L::NV : 4;
        for (int32_t i = 0; i < a.n; i += kFlight * L::kSpan) {
            if (__any(hits & ((1u << kFlight) - 1))) {
                P p[kFlight];
                float number[kFlight][L::VEC];
                static_for<kFlight>([&](auto j) __attribute__((always_inline)) {
                    p[j].load(src, i + j * L::kSpan, g.t * L::VEC, a.n);
                    numbers_of(i + j * L::kSpan, number[j]);
                });
                static_for<kFlight>([&](auto j) __attribute__((always_inline)) {
                    draw(in, at, last, i + j * L::kSpan + g.t * L::VEC, p[j], number[j]);
                });
            }
            if constexpr (L::RESIDENT)
                hits >>= kFlight;
        }
    };
    // the kept prefix: keys above tau, and `ties` of those equal to it
    constexpr uint32_t kAll = 0xFFFFFFFFu;
    const uint32_t end = E::key(top) + 1;
    uint32_t tau = E::kFirstKey, ties = kAll;
    const auto cut_at = [&](uint32_t key, float need) __attribute__((always_inline)) {
        // equal classes until a mass of `need`: at least one
        const float many = ceilf(need / exp_fast(x_of(E::from_key(key))));
        const uint32_t take = many >= 4.0e9f ? kAll : many > 1.0f ? (uint32_t)many : 1u;
        ties = key == tau ? min(take, ties) : take;
        tau = key;
    };
    const Cmp all = E::from_key(E::kFirstKey);
    if (unfiltered) {
        if constexpr (L::RESIDENT && PLAIN)
            static_for<L::NV / kAhead>([&](auto B) __attribute__((always_inline)) {
                constexpr int j0 = decltype(B)::value * kAhead;
                Numbers number;
                if (j0 * L::kSpan >= a.n)
                    return;
                if constexpr (j0 > 0)
                    static_for<kAhead>([&](auto j) __attribute__((always_inline)) {
                        numbers_of((j0 + j) * L::kSpan, number[j]);
                    });
                static_for<kAhead>([&](auto j) __attribute__((always_inline)) {
                    row.template again<j0 + decltype(j)::value>();
                    const int32_t i = (j0 + j) * L::kSpan + g.t * L::VEC;
                    if constexpr (j0 > 0)
                        draw(E::lowest(), all, INT32_MAX, i, row.piece[j0 + j], number[j]);
                    else
                        draw(E::lowest(), all, INT32_MAX, i, row.piece[j], early[j]);
                });
            });
        else
            draw_streamed(all, E::lowest(), INT32_MAX);
        finish(g, first_class, x_loaded);
        return;
    }
    uint32_t *fill = &fills[gi];
    if constexpr (kLists) {
        uint64_t *list = lists[gi];
        uint32_t lo = E::kFirstKey;
        const uint32_t lanes = by_k ? top_k : min(kNucleusLanes, (uint32_t)G / 2);
        if ((by_k || by_p) && lanes <= (uint32_t)G)
            lo = max(lo, group_mth(g, mine > E::lowest() ? E::key(mine) : 0, lanes,
                                   (uint32_t *)list));
        while (by_k || by_p) {
            const uint32_t found = collect<TYPE, L>(g, row, most, E::from_key(lo), list, fill);
            if (found > (uint32_t)L::kList) {
                if constexpr (G > kWave)
                    if (by_k && (uint32_t)top_k < found) {    // the k-th key, or nearly
                        const uint32_t enough = top_k <= L::kList ? L::kList : 0;
                        const auto at = narrow<TYPE, L, uint32_t>(
                            g, row, most, {lo, end, 0, found}, top_k, enough, (uint32_t *)list,
                            [](Cmp) { return 1u; });
                        lo = at.lo;
                        if (at.before + at.here <= enough)
                            continue;
                        tau = lo;
                        ties = top_k - at.before;
                    }
                break;
            }
            const bool counted = found <= (uint32_t)kCounted;
            uint64_t *sorted = counted ? placed[gi] : list;
            if (counted)
                place_entries(g, list, found, sorted, numbers[gi],
                              [&](uint64_t x) { return noise[class_of(x)]; });
            else
                sort_entries(g, list, found);
            const uint32_t n = by_k ? min(found, (uint32_t)top_k) : found;
            // by the block, or by its first wave; whether the list reaches the target
            const auto draw_listed = [&](auto &h, uint32_t width) __attribute__((always_inline)) {
                // sums of w before each entry: a run of entries a lane
                const uint32_t run = (n + width - 1) / width, e0 = min(n, g.t * run),
                               e1 = min(n, e0 + run);
                float w = 0.0f, total;
                for (uint32_t e = e0; e < e1; ++e)
                    w += exp_fast(x_of(E::from_key(key_of(sorted[e]))));
                float before = h.scan(w, total);
                const float target = top_p * (by_k ? total : row_mass);
                if (by_p && !by_k && total < target && lo != E::kFirstKey)
                    return false;
                for (uint32_t e = e0; e < e1; ++e) {
                    const float x = x_of(E::from_key(key_of(sorted[e])));
                    const float we = exp_fast(x);
                    if (e == 0 || ((!by_p || before < target) && x >= floor_x)) {
                        const int32_t cls = class_of(sorted[e]);
                        sum.s += we;
                        const float score = x + (counted ? numbers[gi][e] : noise[cls]);
                        if (score > best || (score == best && cls < best_class)) {
                            best = score;
                            best_x = x;
                            best_class = cls;
                        }
                    }
                    before += we;
                }
                finish(h, [&] { return class_of(sorted[0]); }, x_listed);
                return true;
            };
            bool drawn = false;
            if (G > kWave && n <= kWave) {
                if (g.t < kWave) {
                    Group<kWave> h(g.t, nullptr);
                    drawn = draw_listed(h, kWave);
                }
                if (by_p && !by_k) {                      // (a top-k's list suffices)
                    if (g.t == 0)
                        *fill = drawn;
                    g.barrier();
                    drawn = *fill;
                } else {
                    drawn = true;
                }
            } else {
                drawn = draw_listed(g, G);
            }
            if (drawn)
                return;
            if (G > kWave || lo == E::kFirstKey)
                break;
            lo = E::kFirstKey;                            // a wave's list holds the row
        }
    }

    if constexpr (G < kWave && !PLAIN) {
        // by bisection: classes and mass from a key on
        const auto measure = [&](Cmp at, uint32_t &count, float &mass)
            __attribute__((always_inline)) {
            count = 0;
            mass = 0.0f;
            row.each([&](auto, int32_t, const P &p) {
#pragma unroll
                for (int u = 0; u < L::VEC; ++u)
                    if (p.get(u) >= at) {
                        ++count;
                        mass += exp_fast(x_of(p.get(u)));
                    }
            });
            count = g.reduce(count, Add());
            mass = g.reduce(mass, Add());
        };
        uint32_t count, classes = 0;
        float mass, above = 0.0f, target = 0.0f;
        measure(all, count, mass);
        const bool cut = by_k && count > (uint32_t)top_k;
        uint32_t lo = E::kFirstKey, hi = end;
        while (cut && hi - lo > 1) {                      // count(>= lo) >= k > count(>= hi)
            const uint32_t mid = lo + (hi - lo) / 2;
            float m;
            measure(E::from_key(mid), count, m);
            if (count >= (uint32_t)top_k) {
                lo = mid;
            } else {
                hi = mid;
                classes = count;
                above = m;
            }
        }
        if (cut) {
            tau = lo;
            ties = top_k - classes;
            mass = above + (float)ties * exp_fast(x_of(E::from_key(tau)));
        }
        if (by_p) {
            target = top_p * mass;
            hi = end;
            above = 0.0f;
            while (hi - lo > 1) {                         // mass(>= lo) >= target > mass(>= hi)
                const uint32_t mid = lo + (hi - lo) / 2;
                measure(E::from_key(mid), count, mass);
                if (mass >= target) {
                    lo = mid;
                } else {
                    hi = mid;
                    above = mass;
                }
            }
            cut_at(lo, target - above);
        }
    } else if constexpr (G > kWave && !PLAIN) {
        if (by_p) {
            if (by_k) {                                   // the mass of the first k
                Total<!L::RESIDENT> mass;
                const Cmp at = E::from_key(tau);
                row.template stream<2>([&](int32_t, const P &p) {
                    float part = mass.start();
#pragma unroll
                    for (int u = 0; u < L::VEC; ++u)
                        part += p.get(u) > at || (p.get(u) == at && ties == kAll)
                                    ? exp_fast(x_of(p.get(u))) : 0.0f;
                    mass.add(part);
                });
                row_mass = g.reduce(mass.s, Add());
                if (ties != kAll)
                    row_mass += (float)ties * exp_fast(x_of(at));
            }
            // Classes with w < (1 - p) sum / n together have less than (1 - p) sum: the
            // prefix ends before them.  A sum of all classes is 2^51 in fixed point; those
            // of a tau that a top-k cuts stay out of it: equal classes beyond the k-th, of
            // any number, are not of the sum.
            const double unit = uniform(0x1p51 / (double)row_mass);
            const Mass goal = uniform(max((Mass)(top_p * 0x1p51f), (Mass)1));
            const bool cut = ties != kAll;
            const uint32_t least = tau + cut;
            uint32_t lo = least;
            if constexpr (TYPE != kI32)
                lo = max(lo, E::key(top + logf((1.0f - top_p) * row_mass / (float)a.n) *
                                               temperature) - 1);
            Range<Mass> at = {lo, lo + 1, 0, 0};
            if (lo != end)                                // (0 past the largest integer)
                at = narrow<TYPE, L, Mass>(
                    g, row, most, {lo, end, 0, kUnknown}, goal, 0, (Mass *)lists[gi],
                    [&](Cmp v) __attribute__((always_inline)) {
                        const float w = __builtin_amdgcn_exp2f(E::minus(v, top) * c);
                        return to_mass(fminf(w, 1.0f), unit);
                    });
            const float need = (float)((double)(goal - min(at.before, goal)) / unit);
            if (at.here) {
                cut_at(at.lo, need);
            } else if (cut && lo == least) {
                cut_at(tau, need);                        // the goal is among tau's classes
            } else {                                      // rounding left the goal outside
                tau = at.lo;
                ties = kAll;
            }
        }
    }
    if (min_p > 0.0f) {                                   // as a key: x grows with it
        uint32_t no = tau - 1, yes = end - 1;
        while (yes - no > 1) {
            const uint32_t mid = no + (yes - no) / 2;
            if (x_of(E::from_key(mid)) >= floor_x)
                yes = mid;
            else
                no = mid;
        }
        if (yes > tau)
            ties = kAll;
        tau = yes;
        if (floor_x > 0.0f)                               // none: the first class alone
            ties = 1;
    }
    const Cmp at = E::from_key(tau);
    int32_t last = INT32_MAX;                             // the last kept class equal to tau
    if constexpr (G > kWave && !PLAIN) {
        // the kept classes in a list, if they are few: a list of many takes longer to
        // fill, a piece of every lane at a time, than the row to be read again
        uint64_t *list = lists[gi];
        const uint32_t pieces = g.reduce((uint32_t)__popc(pieces_from<L>(most, at)), Add());
        uint32_t found = 0xFFFFFFFFu;
        if (pieces <= (uint32_t)G)
            found = collect<TYPE, L>(g, row, most, at, list, fill);
        if (found <= (uint32_t)L::kList) {
            if (ties != kAll) {
                sort_entries(g, list, found);
                uint32_t above = 0;
                for (uint32_t e = g.t; e < found; e += G)
                    above += key_of(list[e]) > tau;
                above = g.reduce(above, Add());
                found = above + min(ties, found - above);
            }
            // The list's order is that of its atomics: its sum in integers, whose order
            // does not matter.  Units of 2^-40: 4096 weights from 1 down, within 2^-29 of
            // their sum.
            uint64_t units = 0;
            for (uint32_t e = g.t; e < found; e += G) {
                const float x = x_of(E::from_key(key_of(list[e])));
                const int32_t cls = class_of(list[e]);
                const float score = x + noise[cls];
                units += (uint64_t)(exp_fast(x) * 0x1p40f + 0.5f);
                if (score > best || (score == best && cls < best_class)) {
                    best = score;
                    best_x = x;
                    best_class = cls;
                }
            }
            units = g.reduce(units, Add());
            sum.s = g.t == 0 ? (float)units * 0x1p-40f : 0.0f;
            finish(g, first_class, x_listed);
            return;
        }
    }
    if (ties != kAll) {
        uint32_t seen = 0;
        int32_t equal = -1;
        row.stream([&](int32_t i, const P &p) {
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
    // the largest logit below tau's (no element has the key of -0)
    uint32_t below = tau - 1;
    if (TYPE != kI32 && below == 0x7FFFFFFFu >> E::kShift)
        --below;
    draw_streamed(at, E::from_key(below), last);
    finish(g, first_class, x_loaded);
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
            const bool plain = !a.top_ks && !a.top_ps && !a.min_ps && a.top_p >= 1.0f &&
                               !(a.min_p > 0.0f) && (a.top_k == 0 || a.top_k >= n);
            return in_launches(a, L::kBlock, L::kGroups,
                               [&](const SampleArgs &part, uint32_t blocks) {
                if (plain)
                    k_sample<TYPE, L, true><<<blocks, L::kBlock, 0, stream>>>(part);
                else
                    k_sample<TYPE, L, false><<<blocks, L::kBlock, 0, stream>>>(part);
            });
        });
    });
}

}  // namespace bl
