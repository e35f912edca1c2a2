// Verification of drafted classes against a target's probabilities, from given random
// numbers.
//
// A request's drafts t_0 .. t_{len-1} are walked in order: t_i stands if
// u_i < p_i(t_i) / q_i(t_i), p and q the softmaxes of the target's and the drafter's row;
// after the first that does not, at j, the next class is drawn from max(0, p_j - q_j), or,
// where all stand, from the target's row behind them: the largest log(mass) + Gumbel number.
//
// A row's part in a decision is a reference m, at or just above its largest logit, and the sum s
// of its exponentials relative to it, one pass over the row.  Sums are 32-bit terms in 64-bit
// totals, and the quotient of two is good to kLoose of itself; everything behind them is a
// handful of values a request and taken in 64 bits.  A decision that kLoose could turn is taken
// again with sums in 64 bits (about one draft in 10^5), so accepted drafts and classes are
// those of 64-bit arithmetic.
//
// Draws: p - q = p (1 - e^delta) with delta = log q - log p in 64 bits, since the difference
// of two roundings would decide where p and q are close.  The mass is at most p, so a class
// whose log p + number is below the best so far is done with; the others, a few a wave, take
// the logarithm.
//
// Short rows: a wave walks its request alone, and reads nothing behind the first rejection.
// Long rows: k_verify_rows takes the sums of all rows, in parts where there are few, and
// k_verify_draw has a request's blocks each decide its walk from the sums and draw from their
// part of the last row, and k_verify_pick joins the parts.
#include <float.h>

#include <algorithm>

#include "logit_rows.h"

namespace bl {
namespace {

using namespace rows;

// A lane's reference is set kLead binary orders above its largest logit, and set anew, with its sum
// multiplied to be relative to it, where a logit is above it: every 2.8 (in powers of e).  With
// the largest itself as reference, the sum of an ascending row is multiplied with every load, and
// the roundings of equal steps add up (2^22 ascending classes: a quotient off by up to 4e-5).
// What a sum is off by, in shares of itself:
//   exponents: three roundings of 2^-24 of each difference on the way of a term from its logit
//   to the row's reference, X + 5.6 in powers of e (a reference that is rounded may be twice as far
//   ahead), X how far the logit is below the largest, whose mean over the terms is at most the
//   logarithm of the number of classes, 20.8: 4.8e-6
//   exponentials: 2^-23 each, one for the term, one a change of reference, one behind all of
//   them, X / 2.8 + 4 of them: 1.4e-6.  32-bit sums of eight terms: 0.5e-6
// that is 6.7e-6 at 2^30 classes, and twice that for two sums.
constexpr float kLead = 4.0f;
constexpr double kLoose = 1.4e-5;

struct Side {
    const char *rows;                   // NULL: drafts without probabilities
    int64_t row_stride, request_stride; // bytes
    int32_t type;
    float temperature;
    const float *temperatures;

    __device__ const char *row(int64_t r, int32_t i) const
    {
        return rows + r * request_stride + i * row_stride;
    }
    // 1 / T in 64 bits, within what keeps masked terms zero; 0 where T <= 0 (or is a NaN)
    __device__ double inverse_of(int64_t r) const
    {
        const float t = temperatures ? temperatures[r] : temperature;
        return t > 0.0f ? fmin(1.0 / (double)fminf(t, 0x1p120f), 0x1p126) : 0.0;
    }
};

// A row's (or a part's) reference (-inf: no logit; in greedy rows and beside +inf, the largest
// logit itself; every type's values are exact in 64 bits), the first class that has it (of greedy
// rows) and the sum of exponentials relative to it.
struct Stat {
    double m, s;
    int32_t first;
};
constexpr double kInf = __builtin_inf();

// The best class of a part of a draw, by how much its score may be off, and the most that
// any other class's may be.
struct Best {
    double score, off, other;
    int64_t cls;
};

// Where a request's walk ended (or kLeftOpen), the target's row there, and what is drawn from.
struct Walk {
    Stat p;
    int32_t j, less;
};

struct VerifyArgs {
    Side target, draft;
    int64_t n_requests;
    int32_t n, drafts;
    const int32_t *drafted, *lengths;
    const float *uniform, *noise;
    int64_t noise_stride;
    int32_t *accepted, *token;
    float *log_prob;
    // long rows
    Stat *stats;                        // [request][drafts + 1][2][parts]
    int32_t *rejected;                  // [request]: a draft known to be rejected
    struct Walk *walks;                 // [request]
    Best *bests;                        // [request][draw_parts]
    int32_t parts, part, draw_parts, draw_part;

    __device__ int32_t length(int64_t r) const
    {
        return lengths ? min(max(lengths[r], 0), drafts) : drafts;
    }
    __device__ Stat *stat(int64_t r, int32_t i, int side) const
    {
        return stats + ((r * (drafts + 1) + i) * 2 + side) * parts;
    }
};

template <class F>
__device__ __forceinline__ auto by_type(int type, F f)
{
    switch (type) {
    case kI32: return f(std::integral_constant<int, kI32>());
    case kF32: return f(std::integral_constant<int, kF32>());
    case kF16: return f(std::integral_constant<int, kF16>());
    default: return f(std::integral_constant<int, kBf16>());
    }
}

// An element's value, -inf where it is masked.  (Types are told apart here and in the loops over
// rows alone: what is behind them is there once.)
__device__ __forceinline__ double value_at(const char *row, int type, int64_t i)
{
    return by_type(type, [&](auto T) __attribute__((always_inline)) {
        constexpr int TYPE = decltype(T)::value;
        const auto v = load_one<TYPE>(row, i);
        return v > Elem<TYPE>::lowest() ? (double)v : -kInf;
    });
}
// v - m, m the row's reference: 0 at it, -inf for masked values and, beside a +inf, for all others.
__device__ __forceinline__ double below(double v, double m) { return v == m ? 0.0 : v - m; }

// Elements from class i on of a row of n, those of [i, hi) and the rest masked; returns the class
// of the first.  Near the row's end it loads the last VEC of it instead, without a branch a
// lane: such branches, unrolled, took the registers of all that follows.
template <int TYPE, int VEC>
__device__ __forceinline__ int32_t load_end(Piece<TYPE, VEC> &p, const char *row, int32_t i,
                                            int32_t hi, int32_t n)
{
    constexpr int B = Elem<TYPE>::kBytes;
    if (n < VEC) {                                        // (in the whole wave)
        p.fill_masked();
        if (i == 0)
            p.load(row, 0, 0, hi);
        return i;
    }
    const int32_t at = min(i, n - VEC);
    __builtin_memcpy(p.w, row + (int64_t)at * B, sizeof p.w);
#pragma unroll
    for (int u = 0; u < VEC; ++u)
        if (at + u < i || at + u >= hi)
            p.mask(u);
    return at;
}

// f(first class, piece) over [lo, hi) of a row of n, FLIGHT pieces in flight a lane.
template <int TYPE, int G, int VEC, int FLIGHT, class F>
__device__ __forceinline__ void over(const char *row, int32_t lo, int32_t hi, int32_t n, int t, F f)
{
    typedef Piece<TYPE, VEC> P;
    int32_t i = lo;
    for (; i + FLIGHT * G * VEC <= hi; i += FLIGHT * G * VEC) {
        P p[FLIGHT];
        static_for<FLIGHT>([&](auto j) __attribute__((always_inline)) {
            __builtin_memcpy(p[j].w, row + (int64_t)(i + j * G * VEC) * Elem<TYPE>::kBytes
                                         + (uint32_t)(t * VEC * Elem<TYPE>::kBytes), sizeof p[j].w);
        });
        static_for<FLIGHT>([&](auto j) __attribute__((always_inline)) {
            f(i + j * (G * VEC) + t * VEC, p[j]);
        });
    }
#pragma unroll 2
    for (; i < hi; i += G * VEC) {
        P p;
        const int32_t at = load_end(p, row, i + t * VEC, hi, n);
        f(at, p);
    }
}

// The first class of [lo, hi) whose logit is m.
template <int TYPE, int G>
__device__ __forceinline__ int32_t first_at(Group<G> &g, const char *row, int32_t lo, int32_t hi,
                                            int32_t n, typename Elem<TYPE>::Cmp m)
{
    uint32_t first = 0;                                   // ~class
    over<TYPE, G, 4, 1>(row, lo, hi, n, g.t, [&](int32_t i, const Piece<TYPE, 4> &p)
                                                 __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (p.get(u) == m)
                first = max(first, ~(uint32_t)(i + u));
    });
    return (int32_t)~g.reduce(first, Max());
}

// A reference `lead` above v (int32: rounded down), at most the type's largest finite value; +inf
// is its own.
template <int TYPE>
__device__ __forceinline__ typename Elem<TYPE>::Cmp ahead(typename Elem<TYPE>::Cmp v, float lead)
{
    if constexpr (TYPE == kI32) {
        const int32_t up = (int32_t)((uint32_t)v + (uint32_t)fminf(lead, 0x1p30f));
        return up < v ? INT32_MAX : up;
    } else {
        return v > FLT_MAX ? v : fminf(v + lead, FLT_MAX);
    }
}

// Stat of [lo, hi) of a row of n at 1 / T (0: greedy).
template <int TYPE, int G>
__device__ __forceinline__ Stat stat_of(Group<G> &g, const char *row, int32_t lo, int32_t hi,
                                        int32_t n, double inverse)
{
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    constexpr int VEC = 16 / E::kBytes;
    const float c = (float)(inverse * 1.4426950408889634);
    const float lead = inverse > 0.0 ? kLead / c : 0.0f;
    Cmp m = E::lowest();
    double s = 0.0;
    over<TYPE, G, VEC, 4>(row, lo, hi, n, g.t, [&](int32_t, const Piece<TYPE, VEC> &p)
                                                   __attribute__((always_inline)) {
        Cmp vm = E::lowest();
#pragma unroll
        for (int u = 0; u < VEC; ++u) {
            const Cmp v = p.get(u);
            vm = v > vm ? v : vm;
        }
        if (vm > m) {
            const Cmp old = m;
            m = ahead<TYPE>(vm, lead);
            if (s > 0.0)
                s *= (double)__builtin_amdgcn_exp2f(E::minus(old, m) * c);
        }
        float part = 0.0f;
#pragma unroll
        for (int u = 0; u < VEC; ++u) {
            const Cmp v = p.get(u);
            // (masked: -inf or, of two of them or a NaN, no number, which the maximum drops)
            part += __builtin_amdgcn_exp2f(fmaxf(E::minus(v, m), -FLT_MAX) * c);
        }
        s += (double)part;
    });
    const Cmp most = g.reduce(m, Max());
    if (!(most > E::lowest()))
        return {-kInf, 0.0, 0};
    Stat out = {(double)most, 0.0, 0};
    if (inverse == 0.0) {
        out.first = first_at<TYPE, G>(g, row, lo, hi, n, most);
        return out;
    }
    if (E::to_float(most) == __builtin_inff()) {          // shared by those that have it
        s = 0.0;
        over<TYPE, G, VEC, 1>(row, lo, hi, n, g.t, [&](int32_t, const Piece<TYPE, VEC> &p)
                                                       __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < VEC; ++u)
                s += p.get(u) == most ? 1.0 : 0.0;
        });
    } else if (s > 0.0) {
        s *= (double)__builtin_amdgcn_exp2f(E::minus(m, most) * c);
    }
    out.s = g.reduce(s, Add());
    return out;
}

template <int G>
__device__ __forceinline__ Stat stat_of(Group<G> &g, const char *row, int type, int32_t lo,
                                        int32_t hi, int32_t n, double inverse)
{
    return by_type(type, [&](auto T) __attribute__((always_inline)) {
        return stat_of<decltype(T)::value, G>(g, row, lo, hi, n, inverse);
    });
}

// Sums of parts, relative to the largest of them, by 16 lanes; each gets it.
constexpr int kJoin = 16;
__device__ __forceinline__ Stat join(const Stat *parts, int32_t count, double inverse)
{
    if (count == 1)
        return parts[0];
    const int lane = threadIdx.x % kJoin;
    double m = -kInf, s = 0.0;
    int32_t first = 0;
    for (int32_t k = lane; k < count; k += kJoin)
        if (parts[k].m > m) {                             // (the lane's parts ascend)
            m = parts[k].m;
            first = parts[k].first;
        }
    const double most = wave_reduce<kJoin>(m, Max());
    const uint32_t no = m == most && most > -kInf ? ~(uint32_t)first : 0u;
    for (int32_t k = lane; k < count; k += kJoin)
        if (parts[k].s > 0.0)
            s += parts[k].s * exp(below(parts[k].m, most) * inverse);
    return {most, wave_reduce<kJoin>(s, Add()), (int32_t)~wave_reduce<kJoin>(no, Max())};
}

enum : int { kRejected = 0, kAccepted = 1, kOpen = 2 };

// Whether draft i of request r needs the sum of its row of the drafter.
__device__ __forceinline__ bool has_row(const VerifyArgs &a, double inverse_q)
{
    return a.draft.rows && inverse_q > 0.0;
}

// The decision on draft i of request r from its rows' stats, as far as sums that are off by
// `loose` allow.
__device__ __forceinline__ int decide(const VerifyArgs &a, int64_t r, int32_t i,
                                      double inverse_p, double inverse_q, const Stat &p,
                                      const Stat &q, double loose)
{
    const int64_t at = r * a.drafts + i;
    const int32_t t = a.drafted[at];
    if (t < 0 || t >= a.n || p.m == -kInf)
        return kRejected;
    if (inverse_p == 0.0)
        return t == p.first ? kAccepted : kRejected;
    const double x = below(value_at(a.target.row(r, i), a.target.type, t), p.m);
    if (x == -kInf)
        return kRejected;
    // p / q = e^(x - y) s_q / s_p
    double ratio = x * inverse_p, sums = 1.0 / p.s;
    if (has_row(a, inverse_q)) {
        const double v = value_at(a.draft.row(r, i), a.draft.type, t);
        const double y = v == -kInf ? v : below(v, q.m) * inverse_q;
        ratio = y == -kInf ? kInf : ratio - y;
        sums = q.s / p.s;
    }
    ratio = ratio == kInf ? kInf : exp(ratio) * sums;     // (no mass in q at all: s_q is 0)
    const double u = a.uniform[at];
    if (fabs(u - ratio) <= loose * ratio && ratio < kInf)
        return kOpen;
    return u < ratio ? kAccepted : kRejected;
}

// Whether decide() will certainly reject, in 32 bits with a thousandth to spare.  Never where the
// drafter's row has no mass at the draft: p / q is infinite then, while of a row without any (its
// largest -inf, its sum zero) the steps below would make zero.
__device__ __forceinline__ bool surely_rejected(const VerifyArgs &a, int64_t r, int32_t i,
                                                double inverse_p, double inverse_q, const Stat &p,
                                                const Stat &q)
{
    const int64_t at = r * a.drafts + i;
    const int32_t t = a.drafted[at];
    if (t < 0 || t >= a.n || p.m == -kInf)
        return true;
    if (inverse_p == 0.0)
        return t != p.first;
    // (exponents of 10^5 cancel: their difference comes before its rounding)
    double e = below(value_at(a.target.row(r, i), a.target.type, t), p.m) * inverse_p;
    float sums = -__builtin_amdgcn_logf((float)p.s);
    if (has_row(a, inverse_q)) {
        const double v = value_at(a.draft.row(r, i), a.draft.type, t);
        if (v == -kInf)
            return false;
        e -= below(v, q.m) * inverse_q;
        sums += __builtin_amdgcn_logf((float)q.s);
    }
    const float log_ratio = (float)e * kLog2e + sums;
    // (a NaN, of drafts beside +inf in both rows, is not sure)
    return a.uniform[at] > __builtin_amdgcn_exp2f(log_ratio) * 1.001f + 1e-30f;
}

// What the next class is drawn from: the target's row, less the drafter's (kRow), less the
// draft (kOne), or as it is.
enum : int { kWhole = 0, kRow = 1, kOne = 2 };
struct Draw {
    const char *p, *q;
    const float *noise;
    int p_type, q_type, less;
    int32_t n, drafted;
    double pm, qm, inverse_p, inverse_q, log_sums;        // log(s_p / s_q)
};

__device__ __forceinline__ void merge(Best &a, const Best &b)
{
    const bool other = b.score > a.score || (b.score == a.score && b.cls < a.cls);
    const Best low = other ? a : b;
    if (other)
        a = {b.score, b.off, fmax(a.other, b.other), b.cls};
    else
        a.other = fmax(a.other, b.other);
    if (low.score > -kInf)
        a.other = fmax(a.other, low.score + low.off);
}

constexpr int64_t kNoClass = INT64_MAX;
__device__ __forceinline__ Best nothing()
{
    return {-kInf, 0.0, -kInf, kNoClass};
}

// The best of the group's lanes; every lane gets it.
template <int G>
__device__ __forceinline__ Best join(Group<G> &g, const Best &mine)
{
    Best b;
    b.score = g.reduce(mine.score, Max());
    const int64_t no = mine.score == b.score ? ~mine.cls : INT64_MIN;
    b.cls = ~g.reduce(no, Max());
    const bool won = mine.score == b.score && mine.cls == b.cls;
    b.off = g.reduce(won ? mine.off : 0.0, Max());
    double other = mine.other;
    if (!won && mine.score > -kInf)
        other = fmax(other, mine.score + mine.off);
    b.other = g.reduce(other, Max());
    return b;
}

// A class's place in a draw: x = (l - m) / T of the target, y of the drafter, its number.
__device__ __forceinline__ void offer(Best &best, const Draw &d, int32_t cls, double x, double y,
                                      double number)
{
    Best one = {x + number, 0.0, -kInf, cls};
    if (d.less == kOne && cls == d.drafted)
        return;
    if (d.less == kRow && y > -kInf) {
        const double delta = y - x + d.log_sums;          // log(q / p)
        if (!(delta < 2 * kLoose))
            return;
        if (delta > -2 * kLoose) {                        // p > q, or not, by less than 4 kLoose
            const double most = one.score - 9.7;          // log(4 kLoose), rounded up
            if (most > best.other)
                best.other = most;
            return;
        }
        const float w = -expm1f((float)delta);
        one.score += (double)logf(w);
        one.off = kLoose / (double)w;
    }
    if (one.score > -kInf)                     // (no NaN either)
        merge(best, one);
}

// The group's best of classes [lo, hi).  A lane bounds 8 classes by x + number, which no mass
// below p changes upwards, and evaluates its best of them, all lanes at once, while any is above
// what the wave has: two or three times for the first 512 classes, then seldom.  The values are
// loaded again for that (p's are in the L1), which is what keeps the loop small.
template <int G>
__device__ __forceinline__ Best draw_part(Group<G> &g, const Draw &d, int32_t lo, int32_t hi)
{
    constexpr int V = 4, kFlight = 2, N = kFlight * V;
    const float inv = (float)d.inverse_p;
    Best best = nothing();
    float bound = -__builtin_inff();                      // the wave's best, less what it is off
    for (int32_t base = lo; base < hi; base += N * G) {
        float most[N];
        int32_t at[kFlight];
        uint32_t open = 0;                                // not evaluated, and not below the bound
        by_type(d.p_type, [&](auto T) __attribute__((always_inline)) {
            constexpr int TYPE = decltype(T)::value;
            typedef Elem<TYPE> E;
            const auto m = (typename E::Cmp)d.pm;
            Piece<TYPE, V> p[kFlight];
            Piece<kF32, V> z[kFlight];
            const char *numbers = reinterpret_cast<const char *>(d.noise);
            if (base + N * G <= hi) {
#pragma unroll
                for (int j = 0; j < kFlight; ++j) {
                    at[j] = base + j * G * V + g.t * V;
                    __builtin_memcpy(p[j].w, d.p + (int64_t)at[j] * E::kBytes, sizeof p[j].w);
                    __builtin_memcpy(z[j].w, numbers + (int64_t)at[j] * 4, sizeof z[j].w);
                }
            } else {
#pragma unroll
                for (int j = 0; j < kFlight; ++j) {
                    at[j] = load_end(p[j], d.p, base + j * G * V + g.t * V, hi, d.n);
                    load_end(z[j], numbers, base + j * G * V + g.t * V, hi, d.n);
                }
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const auto v = p[k / V].get(k % V);
                const float number = z[k / V].get(k % V);
                const float x = v == m ? 0.0f : E::minus(v, m) * inv;
                // (rounded: a millionth of what it is made of)
                most[k] = x + number + (fabsf(x) + fabsf(number)) * 1e-6f;
                open |= (uint32_t)(v > E::lowest() && !(most[k] < bound)) << k;
            }
        });
#pragma unroll 1
        while (__any(open)) {
            float top = -__builtin_inff();
            int32_t i = -1;
            uint32_t own = 0;
#pragma unroll
            for (int k = 0; k < N; ++k) {                 // (NaNs too: x or number infinite)
                const bool more = (open >> k & 1) && (i < 0 || !(most[k] <= top));
                top = more ? most[k] : top;
                i = more ? at[k / V] + k % V : i;
                own = more ? 1u << k : own;
            }
            if (i >= 0) {
                open &= ~own;
                const double x = below(value_at(d.p, d.p_type, i), d.pm) * d.inverse_p;
                double y = 0.0;
                if (d.less == kRow) {
                    const double v = value_at(d.q, d.q_type, i);
                    y = v == -kInf ? v : below(v, d.qm) * d.inverse_q;
                }
                offer(best, d, i, x, y, (double)d.noise[i]);
            }
            float low = (float)(best.score - best.off);
            low -= fabsf(low) * 1e-6f;
            bound = wave_reduce<(G < kWave ? G : kWave)>(fmaxf(low, bound), Max());
#pragma unroll
            for (int k = 0; k < N; ++k)
                open &= ~((uint32_t)(most[k] < bound) << k);
        }
    }
    return join(g, best);
}

// The draw at row j of request r, of which `length` drafts were given.
__device__ __forceinline__ Draw draw_of(const VerifyArgs &a, int64_t r, int32_t j,
                                        int32_t length, double inverse_p, double inverse_q,
                                        const Stat &p, const Stat &q)
{
    Draw d;
    d.p = a.target.row(r, j);
    d.q = nullptr;
    d.noise = a.noise + r * a.noise_stride;
    d.p_type = a.target.type;
    d.q_type = a.draft.type;
    d.n = a.n;
    d.drafted = -1;
    d.pm = p.m;
    d.qm = q.m;
    d.inverse_p = inverse_p;
    d.inverse_q = inverse_q;
    d.log_sums = 0.0;
    d.less = kWhole;
    if (j < length) {
        if (!has_row(a, inverse_q)) {
            d.less = kOne;
            d.drafted = a.drafted[r * a.drafts + j];
        } else if (q.m > -kInf) {
            d.less = kRow;
            d.q = a.draft.row(r, j);
            d.log_sums = log(p.s / q.s);
        }
    }
    return d;
}

// One lane's: what comes back for a request.
__device__ __forceinline__ void answer(const VerifyArgs &a, int64_t r, int32_t j, int32_t token,
                                       double inverse_p, const Stat &p)
{
    a.accepted[r] = j;
    a.token[r] = token;
    if (a.log_prob) {
        float value = token < 0 ? -__builtin_inff() : 0.0f;
        if (token >= 0 && inverse_p > 0.0)
            value = (float)(below(value_at(a.target.row(r, j), a.target.type, token), p.m)
                            * inverse_p - log(p.s));
        a.log_prob[r] = value;
    }
}

// ---- the walk ----
// The first of drafts [base, base + 64), below `length`, that does not stand, or kNone; kLeftOpen
// where 32 bits do not tell.  stats: p and q of each in turn.  By a wave.
constexpr int32_t kNone = -1, kLeftOpen = -2;
__device__ __forceinline__ int32_t walk(const VerifyArgs &a, int64_t r, int32_t base,
                                        int32_t length, double inverse_p, double inverse_q,
                                        const Stat *stats)
{
    const int lane = threadIdx.x % kWave;
    int how = kAccepted;
    if (base + lane < length)
        how = decide(a, r, base + lane, inverse_p, inverse_q, stats[2 * lane], stats[2 * lane + 1],
                     kLoose);
    const uint64_t ends = __ballot(how != kAccepted);
    if (!ends)
        return kNone;
    const int k = __builtin_ctzll(ends);
    return __shfl(how, k) == kOpen ? kLeftOpen : base + k;
}

// The class of a draw, or kLeftOpen: it takes 64 bits, or there is none in what is left of p.
__device__ __forceinline__ int32_t settle(int less, const Best &best)
{
    const bool open = best.cls == kNoClass ||
                      (less == kRow && best.other > -kInf &&
                       best.other >= best.score - best.off);
    return open ? kLeftOpen : (int32_t)best.cls;
}

// A request from the start in 64 bits throughout, by a group: what 32 bits left open, and draws
// without a class.  Rare (a draft or draw in 10^4 or so), and behind everything else, so that
// it takes no registers from what always runs.
template <int G>
__device__ __forceinline__ void redo(Group<G> &g, const VerifyArgs &a, int64_t r)
{
    struct Row {
        const char *p;
        int type;
        double inverse, m, log_s;
        int32_t first;
        __device__ __forceinline__ double value(int64_t i) const          // -inf: masked
        {
            return value_at(p, type, i);
        }
        // log of a class's share
        __device__ __forceinline__ double log_share(int64_t i) const
        {
            const double v = value(i);
            return v == -kInf ? v : (v == m ? 0.0 : v - m) * inverse - log_s;
        }
        __device__ __forceinline__ void take(Group<G> &g, const Side &of, int64_t r, int32_t i, int32_t n)
        {
            p = of.row(r, i);
            type = of.type;
            inverse = of.inverse_of(r);
            m = -kInf;
            uint32_t at = 0;
            for (int32_t k = g.t; k < n; k += G) {
                const double v = value(k);
                if (v > m) {
                    m = v;
                    at = ~(uint32_t)k;
                }
            }
            const double most = g.reduce(m, Max());
            first = (int32_t)~g.reduce(m == most ? at : 0u, Max());
            m = most;
            log_s = 0.0;
            double s = 0.0;
            for (int32_t k = g.t; k < n; k += G)
                s += exp(log_share(k));
            log_s = log(g.reduce(s, Add()));
        }
    };
    const int32_t length = a.length(r);
    Row p, q;
    int32_t j = 0, t = -1;
    bool row_q = false;
    for (;; ++j) {
        p.take(g, a.target, r, j, a.n);
        if (j == length)
            break;
        t = a.drafted[r * a.drafts + j];
        row_q = has_row(a, a.draft.inverse_of(r));
        if (row_q)
            q.take(g, a.draft, r, j, a.n);
        if (t < 0 || t >= a.n)
            break;
        const double log_p = p.log_share(t), log_q = row_q ? q.log_share(t) : 0.0;
        if (!(log_p > -kInf) ||
            !((double)a.uniform[r * a.drafts + j] <
              (log_q == -kInf ? kInf : exp(log_p - log_q))))
            break;
    }
    // from what is left of p or, where no class has more in it, from p
    Best best = nothing();
    const bool masked = p.m == -kInf;
    for (int turn = j < length ? 0 : 1; turn < 2 && !masked; ++turn) {
        const bool rest = turn == 0;
        bool mass = false;
        for (int32_t i = g.t; i < a.n; i += G) {
            const double share = exp(p.log_share(i));
            const double less = !rest ? 0.0 : row_q ? exp(q.log_share(i)) : i == t ? 1.0 : 0.0;
            if (!(share > less))                          // (a NaN: a row of masked logits)
                if (!(rest && row_q && q.m == -kInf && share > 0.0))
                    continue;
            mass = true;
            const double left = rest && !(row_q && q.m == -kInf) ? share - less : share;
            const double score = log(left) + (double)a.noise[r * a.noise_stride + i];
            if (score > -kInf)
                merge(best, {score, 0.0, -kInf, i});
        }
        if (g.reduce((uint32_t)mass, Max()))
            break;
    }
    best = join(g, best);
    if (g.t == 0) {
        const int32_t token = masked ? -1 : best.cls == kNoClass ? p.first : (int32_t)best.cls;
        a.accepted[r] = j;
        a.token[r] = token;
        if (a.log_prob)
            a.log_prob[r] = token < 0 ? -__builtin_inff() : (float)p.log_share(token);
    }
}

// ---- short rows: a wave a request ----
// Rows of up to kManyRows classes: 16 lanes a row, the rows of 32 drafts together, since a wait
// for memory costs more than rows behind a rejection.  Longer ones: a draft's rows at a time.
// (1024 requests of 1024 classes 22 us and 29, of 2048 35 and 37, of 4096 57 and 54.)
constexpr int kShortBlock = 256;
constexpr int32_t kManyRows = 2048;

template <int G>
__global__ __launch_bounds__(kShortBlock, 4) void k_verify_short(VerifyArgs a)
{
    constexpr int kGroups = kShortBlock / kWave, kDrafts = G < kWave ? 32 : 1;
    __shared__ Stat all[kGroups][2 * kDrafts];
    const int gi = group_of<kWave>(), lane = threadIdx.x % kWave;
    Group<kWave> g(lane, nullptr);
    Group<G> own(lane % G, nullptr);
    Stat *stats = all[gi];
    for (int64_t r = (int64_t)blockIdx.x * kGroups + gi; r < a.n_requests;
         r += (int64_t)gridDim.x * kGroups) {
        const double inverse_p = uniform(a.target.inverse_of(r));
        const double inverse_q = uniform(a.draft.inverse_of(r));
        const int32_t length = uniform(a.length(r));
        const bool both = has_row(a, inverse_q) && inverse_p > 0.0;
        int32_t j = -1, base = 0;
        for (;; base += kDrafts) {
            const int32_t count = min(kDrafts, length + 1 - base);     // (of the target's rows)
            for (int32_t u = lane / G; u < 2 * count; u += kWave / G) {
                const int32_t i = base + u / 2;
                const bool q = u & 1;
                if (q && (!both || i == length))
                    continue;
                const Stat one = stat_of(own, q ? a.draft.row(r, i) : a.target.row(r, i),
                                         q ? a.draft.type : a.target.type, 0, a.n, a.n,
                                         q ? inverse_q : inverse_p);
                if (own.t == 0)
                    stats[u] = one;
            }
            wave_sync();
            j = walk(a, r, base, min(length, base + kDrafts), inverse_p, inverse_q, stats);
            if (j == kNone && length < base + kDrafts)
                j = length;
            if (j != kNone)
                break;
            wave_sync();
        }
        int32_t token = j == kLeftOpen ? kLeftOpen : -1;
        if (j >= 0) {
            const Stat p = stats[2 * (j - base)], q = stats[2 * (j - base) + 1];
            wave_sync();
            if (p.m > -kInf) {
                if (inverse_p > 0.0) {
                    const Draw d = draw_of(a, r, j, length, inverse_p, inverse_q, p, q);
                    token = settle(d.less, draw_part(g, d, 0, a.n));
                } else {
                    token = p.first;
                }
            }
            if (lane == 0 && token != kLeftOpen)
                answer(a, r, j, token, inverse_p, p);
        }
        if (token == kLeftOpen)
            redo(g, a, r);
    }
}

// ---- long rows ----

__global__ __launch_bounds__(256) void k_verify_clear(VerifyArgs a)
{
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < a.n_requests;
         r += (int64_t)gridDim.x * 256)
        a.rejected[r] = INT32_MAX;
}

// The stats of row i of request r, target's and drafter's, or of a part of them.  Whole rows
// (WHOLE): rows i of all requests before rows i + 1 of any, and a row behind a draft that is
// known to be rejected by then is left out: nobody asks for it.
template <int G, bool WHOLE>
__global__ __launch_bounds__(G, 8) void k_verify_rows(VerifyArgs a)
{
    __shared__ Scratch scratch;
    __shared__ int32_t known;
    Group<G> g(threadIdx.x, &scratch);
    const int64_t units = a.n_requests * (a.drafts + 1) * a.parts;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int64_t row = WHOLE ? unit : unit / a.parts;
        const int32_t part = WHOLE ? 0 : (int32_t)(unit - row * a.parts);
        const int32_t i = (int32_t)(row / a.n_requests);
        const int64_t r = row - i * a.n_requests;
        const int32_t length = a.length(r);
        if (i > length)
            continue;
        if (WHOLE) {
            // one lane asks, so that the block has one answer
            if (g.t == 0)
                known = __hip_atomic_load(&a.rejected[r], __ATOMIC_RELAXED,
                                          __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            const bool left_out = known < i;
            __syncthreads();
            if (left_out)
                continue;
        }
        const int32_t lo = part * a.part, hi = min(a.n, lo + a.part);
        const double inverse_p = a.target.inverse_of(r), inverse_q = a.draft.inverse_of(r);
        Stat p, q = {-kInf, 0.0, 0};
        const bool both = i < length && has_row(a, inverse_q) && inverse_p > 0.0;
        for (int side = 0; side <= (int)both; ++side) {
            const Stat one = stat_of(g, side ? a.draft.row(r, i) : a.target.row(r, i),
                                     side ? a.draft.type : a.target.type, lo, hi, a.n,
                                     side ? inverse_q : inverse_p);
            (side ? q : p) = one;
        }
        if (g.t == 0) {
            a.stat(r, i, 0)[part] = p;
            a.stat(r, i, 1)[part] = q;
            if (WHOLE && i < length && surely_rejected(a, r, i, inverse_p, inverse_q, p, q))
                atomicMin(&a.rejected[r], i);
        }
    }
}

constexpr int kDrawBlock = 256;

__global__ __launch_bounds__(kDrawBlock, 4) void k_verify_draw(VerifyArgs a)
{
    constexpr int G = kDrawBlock, kDrafts = 64;
    __shared__ Scratch scratch;
    __shared__ int32_t found;
    __shared__ Stat stats[2 * kDrafts];
    Group<G> g(threadIdx.x, &scratch);
    const int64_t units = a.n_requests * a.draw_parts;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int64_t r = unit / a.draw_parts;
        const int32_t part = (int32_t)(unit - r * a.draw_parts);
        const double inverse_p = a.target.inverse_of(r), inverse_q = a.draft.inverse_of(r);
        const int32_t length = a.length(r);
        // the walk, kDrafts at a time: their rows' parts joined by 16 lanes each, then the
        // decisions, which one wave takes (64-bit exponentials in all four: 30 us of 109)
        const bool both = has_row(a, inverse_q) && inverse_p > 0.0;
        int32_t j = -1, base = 0;
        for (;; base += kDrafts) {
            const int32_t count = min(kDrafts, length + 1 - base);
            for (int32_t u = threadIdx.x / kJoin; u < 2 * count; u += G / kJoin) {
                const int32_t i = base + u / 2;
                const bool q = u & 1;
                if (q && (!both || i == length))
                    continue;
                const Stat one = join(a.stat(r, i, q), a.parts, q ? inverse_q : inverse_p);
                if (threadIdx.x % kJoin == 0)
                    stats[u] = one;
            }
            __syncthreads();
            if (threadIdx.x < kWave) {
                j = walk(a, r, base, min(length, base + kDrafts), inverse_p, inverse_q, stats);
                if (j == kNone && length < base + kDrafts)
                    j = length;
                if (threadIdx.x == 0)
                    found = j;
            }
            __syncthreads();
            j = found;
            if (j != kNone)
                break;
        }
        const bool open = j == kLeftOpen;                 // (all of the request's blocks see it)
        Stat p = {-kInf, 0.0, 0}, q = p;
        if (!open) {
            p = stats[2 * (j - base)];
            q = stats[2 * (j - base) + 1];
        }
        __syncthreads();                                  // (the next unit writes them)
        const bool drawn = !open && inverse_p > 0.0 && p.m > -kInf;
        int32_t less = kWhole;
        if (drawn) {
            const Draw d = draw_of(a, r, j, length, inverse_p, inverse_q, p, q);
            const int32_t lo = part * a.draw_part;
            const Best best = draw_part(g, d, lo, min(a.n, lo + a.draw_part));
            if (g.t == 0)
                a.bests[r * a.draw_parts + part] = best;
            less = d.less;
        }
        if (part == 0 && g.t == 0)
            a.walks[r] = {p, j, less};
    }
}

// The parts of a request's draw joined, by a wave.  (A last block that joins them instead needs
// fences between the dies' L2s, one a block: 192 x 131072, 16 blocks a request, 195 us, without 74.)
// A whole block, for what 32 bits left open: 64 lanes took 4 ms more for a row of 131072.
constexpr int kPickBlock = 1024;

__global__ __launch_bounds__(kPickBlock) void k_verify_pick(VerifyArgs a)
{
    __shared__ Scratch scratch;
    __shared__ int32_t picked;
    Group<kPickBlock> g(threadIdx.x, &scratch);
    for (int64_t r = blockIdx.x; r < a.n_requests; r += gridDim.x) {
        if (threadIdx.x < kWave) {
            Group<kWave> wave(threadIdx.x, nullptr);
            const Walk w = a.walks[r];
            const double inverse_p = a.target.inverse_of(r);
            int32_t token = w.j == kLeftOpen ? kLeftOpen : w.p.m == -kInf ? -1 : w.p.first;
            if (token >= 0 && inverse_p > 0.0) {
                Best best = nothing();
                for (int32_t k = wave.t; k < a.draw_parts; k += kWave)
                    merge(best, a.bests[r * a.draw_parts + k]);
                token = settle(w.less, join(wave, best));
            }
            if (threadIdx.x == 0) {
                picked = token;
                if (token != kLeftOpen)
                    answer(a, r, w.j, token, inverse_p, w.p);
            }
        }
        __syncthreads();
        const bool open = picked == kLeftOpen;
        __syncthreads();                                  // (the next request writes it)
        if (open)
            redo(g, a, r);
    }
}

// ---- which form, and its workspace ----
// A wave a request: always up to kShortClasses, and up to kMostShort where requests are enough to
// fill the card; else k_verify_rows and what follows (us, 4 drafts of bfloat16: 1030 classes, 16
// requests 22 and 24, 1400 46 and 72; 1300 classes, 256 requests 30 and 28, 400 30 and 33; 2048
// classes, 400 39 and 34, 600 36 and 39; 4096 classes, 512 51 and 42, 850 56 and 62; of 8
// drafts the border is where it is for 4, of one below: 2048 classes, 256 requests 21 and 24).
// Above 4096 what a wave alone may have to redo in 64 bits (500 us for 8192 classes, in about one
// call of 25 with 1024 requests) costs what is won.
constexpr int32_t kShortClasses = 1024, kMostShort = 4096;
constexpr int kWholeBlock = 1024;

struct Plan {
    bool is_short, whole;
    int32_t parts, part, draw_parts, draw_part;
    size_t rejected, walks, bests, bytes;
};

size_t up(size_t v) { return (v + 255) / 256 * 256; }

// Parts of a row, each a multiple of `unit` classes, for about `want` blocks over `rows` rows.
void split(int64_t rows, int32_t n, int64_t want, int32_t unit, int32_t &parts, int32_t &part)
{
    const int64_t most = ((int64_t)n + unit - 1) / unit;
    const int64_t p = std::min(most, std::max<int64_t>(1, want / rows));
    part = (int32_t)((most + p - 1) / p) * unit;
    parts = (int32_t)(((int64_t)n + part - 1) / part);
}

Plan plan_of(int64_t n_requests, int32_t drafts, int32_t n)
{
    Plan p = {};
    p.is_short = n <= kShortClasses || (n <= kMostShort && n_requests >= n / 6 + 160);
    if (p.is_short || n_requests == 0)
        return p;
    const int64_t rows = n_requests * (drafts + 1);
    // A block of 1024 a row, which skips rows behind a rejection, or blocks of 256 (us, all
    // kernels): 2000 rows of 8192 59 and 39, 5000 87 and 85; 1000 of 65536 94 and 90, 2000 163
    // and 166; 1152 of 131072, four drafts in five standing, 160 and 182.
    p.whole = rows >= 1024 && rows * n >= 1 << 26;
    split(rows, n, p.whole ? 1 : 1024, 4096, p.parts, p.part);
    // (192 rows of 131072, all kernels: 169 us at 1024 blocks, 158 at 2048, 154 at 4096; one
    // row: 23.8, 24.3 and 25.1)
    split(n_requests, n, 2048, 4096, p.draw_parts, p.draw_part);
    p.rejected = up((size_t)rows * 2 * p.parts * sizeof(Stat));
    p.walks = p.rejected + up((size_t)n_requests * 4);
    p.bests = p.walks + up((size_t)n_requests * sizeof(Walk));
    p.bytes = p.bests + (size_t)n_requests * p.draw_parts * sizeof(Best);
    return p;
}

}  // namespace

size_t verify_workspace_bytes(int64_t n_requests, int32_t drafts, int32_t n)
{
    return plan_of(n_requests, drafts, n).bytes;
}

hipError_t launch_verify(const VerifySide &target, const VerifySide &draft, int64_t n_requests,
                         int32_t n, int32_t drafts, const int32_t *drafted,
                         const int32_t *lengths, const float *uniform, const float *noise,
                         int64_t noise_stride, int32_t *accepted, int32_t *token,
                         float *log_prob, void *workspace, hipStream_t stream)
{
    const auto side = [](const VerifySide &s) {
        const int64_t bytes = s.type == kI32 || s.type == kF32 ? 4 : 2;
        return Side{static_cast<const char *>(s.logits), s.row_stride * bytes,
                    s.request_stride * bytes, s.type, s.temperature, s.temperatures};
    };
    VerifyArgs a = {};
    a.target = side(target);
    a.draft = side(draft);
    a.n_requests = n_requests;
    a.n = n;
    a.drafts = drafts;
    a.drafted = drafted;
    a.lengths = lengths;
    a.uniform = uniform;
    a.noise = noise;
    a.noise_stride = noise_stride;
    a.accepted = accepted;
    a.token = token;
    a.log_prob = log_prob;
    const auto grid = [](int64_t blocks) {
        return dim3((uint32_t)std::min<int64_t>(blocks, 1 << 20));
    };
    const Plan p = plan_of(n_requests, drafts, n);
    if (p.is_short) {
        constexpr int kGroups = kShortBlock / kWave;
        if (n <= kManyRows)
            hipLaunchKernelGGL(k_verify_short<16>, grid((n_requests + kGroups - 1) / kGroups),
                               dim3(kShortBlock), 0, stream, a);
        else
            hipLaunchKernelGGL(k_verify_short<64>, grid((n_requests + kGroups - 1) / kGroups),
                               dim3(kShortBlock), 0, stream, a);
        return hipGetLastError();
    }
    char *ws = static_cast<char *>(workspace);
    a.stats = reinterpret_cast<Stat *>(ws);
    a.rejected = reinterpret_cast<int32_t *>(ws + p.rejected);
    a.walks = reinterpret_cast<Walk *>(ws + p.walks);
    a.bests = reinterpret_cast<Best *>(ws + p.bests);
    a.parts = p.parts;
    a.part = p.part;
    a.draw_parts = p.draw_parts;
    a.draw_part = p.draw_part;
    const int64_t units = n_requests * (drafts + 1) * p.parts;
    if (p.whole) {
        hipLaunchKernelGGL(k_verify_clear, grid((n_requests + 255) / 256), dim3(256), 0, stream,
                           a);
        hipLaunchKernelGGL((k_verify_rows<kWholeBlock, true>), grid(units), dim3(kWholeBlock),
                           0, stream, a);
    } else {
        hipLaunchKernelGGL((k_verify_rows<256, false>), grid(units), dim3(256), 0, stream, a);
    }
    if (hipError_t err = hipGetLastError(); err != hipSuccess)
        return err;
    hipLaunchKernelGGL(k_verify_draw, grid(n_requests * p.draw_parts), dim3(kDrawBlock), 0,
                       stream, a);
    if (hipError_t err = hipGetLastError(); err != hipSuccess)
        return err;
    hipLaunchKernelGGL(k_verify_pick, grid(n_requests), dim3(kPickBlock), 0, stream, a);
    return hipGetLastError();
}

}  // namespace bl
