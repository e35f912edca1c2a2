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
// Every filter keeps a prefix of the order, so the kept set is (key > tau) and the
// first classes of (key == tau).  tau comes from bisection on the key: on counts for
// top-k, on sums of w for top-p.
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

template <int TYPE, class L>
__global__ __launch_bounds__(L::kBlock) void k_sample(SampleArgs a)
{
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    typedef Piece<TYPE, L::VEC> P;
    __shared__ Scratch scratch;
    const int64_t r = (int64_t)blockIdx.x * L::kGroups + threadIdx.x / L::G;
    if (r >= a.n_rows)
        return;
    Group<L::G> g(threadIdx.x % L::G, &scratch);
    const char *src = a.logits + r * a.stride;
    const Row<TYPE, L::G, L::NV, L::VEC, L::RESIDENT> row(src, a.n, g.t);
    const float temperature = a.temperatures ? a.temperatures[r] : a.temperature;
    const float top_p = a.top_ps ? a.top_ps[r] : a.top_p;
    const float min_p = a.min_ps ? a.min_ps[r] : a.min_p;
    const int32_t top_k = a.top_ks ? a.top_ks[r] : a.top_k;

    // the first of the order: the lowest class among the largest logits
    Cmp top = E::lowest();
    row.each([&](int, int32_t, const P &p) {
#pragma unroll
        for (int u = 0; u < L::VEC; ++u) {
            const Cmp v = p.get(u);
            top = v > top ? v : top;
        }
    });
    top = g.reduce(top, Max());
    if (!(top > E::lowest())) {                           // nothing to draw from
        if (g.t == 0) {
            a.token[r] = -1;
            if (a.log_prob)
                a.log_prob[r] = -__builtin_inff();
        }
        return;
    }
    uint32_t first = 0;                                   // its ~class
    row.each([&](int, int32_t i, const P &p) {
#pragma unroll
        for (int u = 0; u < L::VEC; ++u)
            if (p.get(u) == top)
                first = max(first, ~(uint32_t)(i + u));
    });
    first = ~g.reduce(first, Max());
    if (!(temperature > 0.0f)) {                          // greedy
        if (g.t == 0) {
            a.token[r] = (int32_t)first;
            if (a.log_prob)
                a.log_prob[r] = 0.0f;
        }
        return;
    }

    const float inv_t = 1.0f / temperature, ftop = E::to_float(top);
    const auto x_of = [&](Cmp v) __attribute__((always_inline)) { return v == top ? 0.0f : (E::to_float(v) - ftop) * inv_t; };
    const auto mass_from = [&](Cmp at) __attribute__((always_inline)) {                  // sum of w over logits >= at
        float sum = 0.0f;
        row.each([&](int, int32_t, const P &p) {
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
        row.each([&](int, int32_t, const P &p) {
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                count += p.get(u) >= at;
        });
        return g.reduce(count, Add());
    };

    // the kept prefix: keys above tau, and `ties` of those equal to it
    const uint32_t end = E::key(top) + 1;
    uint32_t tau = E::kFirstKey, ties = 0xFFFFFFFFu;
    if (top_k > 0 && top_k < a.n && count_from(E::from_key(tau)) > (uint32_t)top_k) {
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
    if (top_p < 1.0f) {
        const Cmp at = E::from_key(tau);
        float target;
        if (ties != 0xFFFFFFFFu) {
            const float above = tau + 1 == end ? 0.0f : mass_from(E::from_key(tau + 1));
            target = top_p * (above + (float)ties * exp_fast(x_of(at)));
        } else {
            target = top_p * mass_from(at);
        }
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
        int32_t mine = -1;
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
                    mine = i + u;
        });
        last = g.reduce(mine, Max());
    }
    const float floor_x = min_p > 0.0f ? logf(min_p) : -__builtin_inff();

    float sum = 0.0f;
    uint64_t best = 0;
    const float *noise = a.noise + r * a.noise_stride;
    row.each([&](int, int32_t i, const P &p) {
#pragma unroll
        for (int u = 0; u < L::VEC; ++u) {
            const Cmp v = p.get(u);
            const float x = x_of(v);
            if ((v > at || (v == at && i + u <= last)) && (x >= floor_x || v == top)) {
                sum += exp_fast(x);
                const float score = x + noise[i + u];
                if (score > -__builtin_inff()) {
                    const uint64_t s = (uint64_t)Elem<kF32>::key(score) << 32 | ~(uint32_t)(i + u);
                    best = s > best ? s : best;
                }
            }
        }
    });
    best = g.reduce(best, Max());
    sum = g.reduce(sum, Add());
    if (g.t == 0) {
        const int32_t token = best ? (int32_t)~(uint32_t)best : (int32_t)first;
        a.token[r] = token;
        if (a.log_prob)
            a.log_prob[r] = x_of(load_one<TYPE>(src, token)) - logf(sum);
    }
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
