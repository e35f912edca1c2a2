// Verification of drafted classes against a target's probabilities, from given random
// numbers.
//
// A request's drafts t_0 .. t_{len-1} are walked in order: t_i stands if
// u_i < p_i(t_i) / q_i(t_i), p and q the softmaxes of the target's and the drafter's row;
// after the first that does not, at j, the next class is drawn from max(0, p_j - q_j), or,
// where all stand, from the target's row behind them: the largest log(mass) + Gumbel number.
//
// A row's part in a decision is its largest logit m and the sum s of its exponentials, one
// pass over the row.  Sums are 32-bit terms in 64-bit totals and good to kLoose of
// themselves; everything behind them is a handful of values a request and taken in 64 bits.
// A decision that kLoose could turn is taken again with sums in 64 bits (about one draft in
// 10^5), so accepted drafts and classes are those of 64-bit arithmetic.
//
// Draws: p - q = p (1 - e^delta) with delta = log q - log p in 64 bits, since the difference
// of two roundings would decide where p and q are close.  The mass is at most p, so a class
// whose log p + number is below the best so far is done with; the others, a few a wave, take
// the logarithm.
//
// Short rows: a wave walks its request alone, and reads nothing behind the first rejection.
// Long rows: k_verify_rows takes the sums of all rows, in parts where there are few, and
// k_verify_draw has a request's blocks each decide its walk from the sums and draw from their
// part of the last row; the last of them joins the parts.
#include <float.h>

#include <algorithm>

#include "logit_rows.h"

namespace bl {
namespace {

using namespace rows;

constexpr double kLoose = 1e-5;

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
    // 1 / T in 64 bits; 0 where T <= 0 (or is a NaN)
    __device__ double inverse_of(int64_t r) const
    {
        const float t = temperatures ? temperatures[r] : temperature;
        return t > 0.0f ? fmin(1.0 / (double)fminf(t, FLT_MAX), 0x1p126) : 0.0;
    }
};

// A row's (or a part's) largest logit, as its bits, the first class that has it (of greedy
// rows) and the sum of exponentials relative to it.
struct Stat {
    uint32_t m;
    int32_t first;
    double s;
};

// The best class of a part of a draw, by how much its score may be off, and the most that
// any other class's may be.
struct Best {
    double score, off, other;
    int64_t cls;
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
    uint32_t *done;                     // [request]: finished parts of the draw
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

template <int TYPE>
__device__ __forceinline__ typename Elem<TYPE>::Cmp cmp_of(uint32_t bits)
{
    typename Elem<TYPE>::Cmp v;
    __builtin_memcpy(&v, &bits, 4);
    return v;
}
template <class T>
__device__ __forceinline__ uint32_t bits_of(T v)
{
    uint32_t b;
    __builtin_memcpy(&b, &v, 4);
    return b;
}

// v - m in 64 bits, m the row's largest: 0 at it, -inf for masked classes and, beside a
// +inf, for all others.
template <int TYPE>
__device__ __forceinline__ double below(typename Elem<TYPE>::Cmp v, typename Elem<TYPE>::Cmp m)
{
    return !(v > Elem<TYPE>::lowest()) ? -__builtin_inf() : v == m ? 0.0 : (double)v - (double)m;
}

__device__ __forceinline__ double below_at(const char *row, int type, int64_t i, uint32_t m)
{
    return by_type(type, [&](auto T) {
        constexpr int TYPE = decltype(T)::value;
        return below<TYPE>(load_one<TYPE>(row, i), cmp_of<TYPE>(m));
    });
}

// f(class, piece) over [lo, hi) of a row, kFlight pieces in flight a lane.
template <int TYPE, int G, int VEC, int FLIGHT, class F>
__device__ __forceinline__ void over(const char *row, int32_t lo, int32_t hi, int t, F f)
{
    for (int32_t i = lo; i < hi; i += FLIGHT * G * VEC) {
        Piece<TYPE, VEC> p[FLIGHT];
        static_for<FLIGHT>([&](auto j) __attribute__((always_inline)) {
            p[j].load(row, i + j * (G * VEC), t * VEC, hi);
        });
        static_for<FLIGHT>([&](auto j) __attribute__((always_inline)) {
            f(i + j * (G * VEC) + t * VEC, p[j]);
        });
    }
}

// The first class of [lo, hi) whose logit is m.
template <int TYPE, class Grp, int G>
__device__ int32_t first_at(Grp &g, const char *row, int32_t lo, int32_t hi,
                            typename Elem<TYPE>::Cmp m)
{
    uint32_t first = 0;                                   // ~class
    over<TYPE, G, 4, 1>(row, lo, hi, g.t, [&](int32_t i, const Piece<TYPE, 4> &p) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (p.get(u) == m)
                first = max(first, ~(uint32_t)(i + u));
    });
    return (int32_t)~g.reduce(first, Max());
}

// Stat of [lo, hi) of a row at 1 / T (0: greedy).
template <int TYPE, int G>
__device__ __forceinline__ Stat stat_of(Group<G> &g, const char *row, int32_t lo, int32_t hi,
                                        double inverse)
{
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    constexpr int VEC = 16 / E::kBytes;
    const float c = (float)(inverse * 1.4426950408889634);
    Cmp m = E::lowest();
    double s = 0.0;
    over<TYPE, G, VEC, 4>(row, lo, hi, g.t, [&](int32_t, const Piece<TYPE, VEC> &p) {
        Cmp vm = E::lowest();
#pragma unroll
        for (int u = 0; u < VEC; ++u) {
            const Cmp v = p.get(u);
            vm = v > vm ? v : vm;
        }
        if (vm > m) {
            if (s > 0.0)
                s *= (double)__builtin_amdgcn_exp2f(E::minus(m, vm) * c);
            m = vm;
        }
        float part = 0.0f;
#pragma unroll
        for (int u = 0; u < VEC; ++u) {
            const Cmp v = p.get(u);
            const float e = __builtin_amdgcn_exp2f(E::minus(v, m) * c);
            part += v > E::lowest() ? e : 0.0f;
        }
        s += (double)part;
    });
    const Cmp most = g.reduce(m, Max());
    Stat out = {bits_of(most), 0, 0.0};
    if (!(most > E::lowest()))
        return out;
    if (inverse == 0.0) {
        out.first = first_at<TYPE, Group<G>, G>(g, row, lo, hi, most);
        return out;
    }
    if (E::to_float(most) == __builtin_inff()) {          // shared by those that have it
        s = 0.0;
        over<TYPE, G, VEC, 1>(row, lo, hi, g.t, [&](int32_t, const Piece<TYPE, VEC> &p) {
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
                                        int32_t hi, double inverse)
{
    return by_type(type, [&](auto T) {
        return stat_of<decltype(T)::value, G>(g, row, lo, hi, inverse);
    });
}

// The sum of a row's exponentials in 64 bits.  (Rare: a call, which takes its own copy of
// the group and ends with a barrier, so that the caller's next reduction finds free slots.)
template <int G>
__device__ __attribute__((noinline)) double exact_sum(Group<G> g, const char *row, int type,
                                                      int32_t n, uint32_t m, double inverse)
{
    double s = 0.0;
    for (int32_t i = g.t; i < n; i += G)
        s += exp(below_at(row, type, i, m) * inverse);
    s = g.reduce(s, Add());
    g.barrier();
    return s;
}

// Sums of parts, relative to the largest of them.
__device__ __forceinline__ Stat join(const Stat *parts, int32_t count, int type, double inverse)
{
    Stat all = parts[0];
    for (int32_t k = 1; k < count; ++k) {
        const Stat one = parts[k];
        by_type(type, [&](auto T) {
            constexpr int TYPE = decltype(T)::value;
            const auto a = cmp_of<TYPE>(all.m), b = cmp_of<TYPE>(one.m);
            if (b > a) {
                all.s = (all.s > 0.0 ? all.s * exp(below<TYPE>(a, b) * inverse) : 0.0) + one.s;
                all.m = one.m;
                all.first = one.first;
            } else if (one.s > 0.0) {
                all.s += one.s * exp(below<TYPE>(b, a) * inverse);
            }
        });
    }
    return all;
}

__device__ __forceinline__ bool is_masked(const Stat &s, int type)
{
    return by_type(type, [&](auto T) {
        constexpr int TYPE = decltype(T)::value;
        return !(cmp_of<TYPE>(s.m) > Elem<TYPE>::lowest());
    });
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
    if (t < 0 || t >= a.n || is_masked(p, a.target.type))
        return kRejected;
    if (inverse_p == 0.0)
        return t == p.first ? kAccepted : kRejected;
    const double x = below_at(a.target.row(r, i), a.target.type, t, p.m);
    if (x == -__builtin_inf())
        return kRejected;
    double log_ratio = x * inverse_p - log(p.s);
    if (has_row(a, inverse_q)) {
        const double y = below_at(a.draft.row(r, i), a.draft.type, t, q.m);
        log_ratio = y == -__builtin_inf() ? __builtin_inf()
                                          : log_ratio - (y * inverse_q - log(q.s));
    }
    const double ratio = exp(log_ratio), u = a.uniform[at];
    if (fabs(u - ratio) <= loose * ratio && ratio < __builtin_inf())
        return kOpen;
    return u < ratio ? kAccepted : kRejected;
}

// decide() with sums in 64 bits, by a group.
template <int G>
__device__ __forceinline__ int decide_exactly(const Group<G> &g, const VerifyArgs &a, int64_t r,
                                              int32_t i, double inverse_p, double inverse_q,
                                              Stat p, Stat q)
{
    p.s = exact_sum(g, a.target.row(r, i), a.target.type, a.n, p.m, inverse_p);
    if (has_row(a, inverse_q) && !is_masked(q, a.draft.type))
        q.s = exact_sum(g, a.draft.row(r, i), a.draft.type, a.n, q.m, inverse_q);
    return decide(a, r, i, inverse_p, inverse_q, p, q, -1.0);
}

// What the next class is drawn from: the target's row, less the drafter's (kRow), less the
// draft (kOne), or as it is.
enum : int { kWhole = 0, kRow = 1, kOne = 2 };
struct Draw {
    const char *p, *q;
    const float *noise;
    int p_type, q_type, less;
    int32_t n, drafted;
    uint32_t pm, qm;
    double inverse_p, inverse_q, log_p, log_q;            // logs of the sums
};

__device__ __forceinline__ void merge(Best &a, const Best &b)
{
    const bool other = b.score > a.score || (b.score == a.score && b.cls < a.cls);
    const Best low = other ? a : b;
    if (other)
        a = {b.score, b.off, fmax(a.other, b.other), b.cls};
    else
        a.other = fmax(a.other, b.other);
    if (low.score > -__builtin_inf())
        a.other = fmax(a.other, low.score + low.off);
}

constexpr int64_t kNoClass = INT64_MAX;
__device__ __forceinline__ Best nothing()
{
    return {-__builtin_inf(), 0.0, -__builtin_inf(), kNoClass};
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
    if (!won && mine.score > -__builtin_inf())
        other = fmax(other, mine.score + mine.off);
    b.other = g.reduce(other, Max());
    return b;
}

// A class's place in a draw: x = (l - m) / T of the target, y of the drafter, its number.
__device__ __forceinline__ void offer(Best &best, const Draw &d, int32_t cls, double x, double y,
                                      double number)
{
    Best one = {x + number, 0.0, -__builtin_inf(), cls};
    if (d.less == kOne && cls == d.drafted)
        return;
    if (d.less == kRow && y > -__builtin_inf()) {
        const double delta = (y - d.log_q) - (x - d.log_p);
        if (!(delta < 2 * kLoose))
            return;
        if (delta > -2 * kLoose) {                        // p > q, or not, by less than 4 kLoose
            const double most = one.score - 10.1;         // log(4 kLoose), rounded up
            if (most > best.other)
                best.other = most;
            return;
        }
        const float w = -expm1f((float)delta);
        one.score += (double)logf(w);
        one.off = kLoose / (double)w;
    }
    if (one.score > -__builtin_inf())                     // (no NaN either)
        merge(best, one);
}

// The group's best of classes [lo, hi).
template <int G>
__device__ __forceinline__ Best draw_part(Group<G> &g, const Draw &d, int32_t lo, int32_t hi)
{
    constexpr int V = 4, kFlight = 2;
    struct Raw {
        uint32_t w[V];
    };
    const auto load = [&](Raw &to, const char *row, int type, int32_t i, int32_t base) {
        by_type(type, [&](auto T) {
            Piece<decltype(T)::value, V> p;
            p.load(row, base, i, hi);
            __builtin_memcpy(to.w, p.w, sizeof p.w);
        });
    };
    Best best = nothing();
    const float inv = (float)d.inverse_p;
    float bound = -__builtin_inff();                      // the wave's best, less what it is off
    for (int32_t base = lo; base < hi; base += kFlight * G * V) {
        Raw p[kFlight], q[kFlight];
        float number[kFlight][V];
#pragma unroll
        for (int j = 0; j < kFlight; ++j) {
            const int32_t from = base + j * G * V, i = g.t * V;
            load(p[j], d.p, d.p_type, i, from);
            if (d.less == kRow)
                load(q[j], d.q, d.q_type, i, from);
            Piece<kF32, V> z;
            z.load(reinterpret_cast<const char *>(d.noise), from, i, hi);
#pragma unroll
            for (int u = 0; u < V; ++u)
                number[j][u] = z.get(u);
        }
#pragma unroll
        for (int j = 0; j < kFlight; ++j) {
            uint32_t in = 0;
            by_type(d.p_type, [&](auto T) {
                constexpr int TYPE = decltype(T)::value;
                Piece<TYPE, V> piece;
                __builtin_memcpy(piece.w, p[j].w, sizeof piece.w);
                const auto m = cmp_of<TYPE>(d.pm);
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    const auto v = piece.get(u);
                    const float x = v == m ? 0.0f : Elem<TYPE>::minus(v, m) * inv;
                    // (rounded: a millionth of what it is made of)
                    const float most = x + number[j][u]
                                       + (fabsf(x) + fabsf(number[j][u])) * 1e-6f;
                    in |= (uint32_t)(v > Elem<TYPE>::lowest() && !(most < bound)) << u;
                }
            });
            if (!__any(in))
                continue;
            const int32_t i = base + j * G * V + g.t * V;
            for (int u = 0; u < V; ++u) {
                if (!(in >> u & 1))
                    continue;
                const auto at = [&](const Raw &raw, int type, uint32_t m) {
                    return by_type(type, [&](auto T) {
                        constexpr int TYPE = decltype(T)::value;
                        Piece<TYPE, V> piece;
                        __builtin_memcpy(piece.w, raw.w, sizeof piece.w);
                        typename Elem<TYPE>::Cmp v = piece.get(0);
#pragma unroll
                        for (int k = 1; k < V; ++k)
                            if (k == u)
                                v = piece.get(k);
                        return below<TYPE>(v, cmp_of<TYPE>(m));
                    });
                };
                float own = number[j][0];
#pragma unroll
                for (int k = 1; k < V; ++k)
                    if (k == u)
                        own = number[j][k];
                const double x = at(p[j], d.p_type, d.pm) * d.inverse_p;
                const double y = d.less == kRow ? at(q[j], d.q_type, d.qm) * d.inverse_q : 0.0;
                offer(best, d, i + u, x, y, (double)own);
            }
            float low = (float)(best.score - best.off);
            low -= fabsf(low) * 1e-6f;
            bound = wave_reduce<(G < kWave ? G : kWave)>(fmaxf(low, bound), Max());
        }
    }
    return join(g, best);
}

// The draw in 64 bits throughout, by a group.
template <int G>
__device__ __attribute__((noinline)) Best draw_exactly(Group<G> g, Draw d)
{
    d.log_p = log(exact_sum(g, d.p, d.p_type, d.n, d.pm, d.inverse_p));
    d.log_q = log(exact_sum(g, d.q, d.q_type, d.n, d.qm, d.inverse_q));
    Best best = nothing();
    for (int32_t i = g.t; i < d.n; i += G) {
        const double p = exp(below_at(d.p, d.p_type, i, d.pm) * d.inverse_p - d.log_p);
        const double q = exp(below_at(d.q, d.q_type, i, d.qm) * d.inverse_q - d.log_q);
        const Best one = {log(p - q) + (double)d.noise[i], 0.0, -__builtin_inf(), i};
        if (p > q && one.score > -__builtin_inf())
            merge(best, one);
    }
    best = join(g, best);
    g.barrier();
    return best;
}

// The class of a draw from the best of all its parts, with what is seldom needed: the draw
// again in 64 bits, from the target's row alone, or the first class of its order.
template <int G>
__device__ __forceinline__ int32_t settle(Group<G> &g, Draw d, Best best)
{
    if (d.less == kRow && best.other > -__builtin_inf() && best.other >= best.score - best.off)
        best = draw_exactly(g, d);
    if (best.cls == kNoClass && d.less != kWhole) {
        d.less = kWhole;
        best = draw_part(g, d, 0, d.n);
    }
    if (best.cls != kNoClass)
        return (int32_t)best.cls;
    return by_type(d.p_type, [&](auto T) {
        constexpr int TYPE = decltype(T)::value;
        return first_at<TYPE, Group<G>, G>(g, d.p, 0, d.n, cmp_of<TYPE>(d.pm));
    });
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
    d.log_p = log(p.s);
    d.log_q = 0.0;
    d.less = kWhole;
    if (j < length) {
        if (!has_row(a, inverse_q)) {
            d.less = kOne;
            d.drafted = a.drafted[r * a.drafts + j];
        } else if (!is_masked(q, a.draft.type)) {
            d.less = kRow;
            d.q = a.draft.row(r, j);
            d.log_q = log(q.s);
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
            value = (float)(below_at(a.target.row(r, j), a.target.type, token, p.m) * inverse_p
                            - log(p.s));
        a.log_prob[r] = value;
    }
}

// ---- short rows: a wave a request ----
constexpr int kShortBlock = 256;

__global__ __launch_bounds__(kShortBlock) void k_verify_short(VerifyArgs a)
{
    constexpr int G = kWave, kGroups = kShortBlock / G;
    const int gi = group_of<G>();
    Group<G> g(threadIdx.x - gi * G, nullptr);
    for (int64_t r = (int64_t)blockIdx.x * kGroups + gi; r < a.n_requests;
         r += (int64_t)gridDim.x * kGroups) {
        const double inverse_p = uniform(a.target.inverse_of(r));
        const double inverse_q = uniform(a.draft.inverse_of(r));
        const int32_t length = uniform(a.length(r));
        int32_t j = 0;
        Stat p, q = {0, 0, 0.0};
        for (;; ++j) {
            const bool both = j < length && has_row(a, inverse_q) && inverse_p > 0.0;
            for (int side = 0; side <= (int)both; ++side) {
                const Side &of = side ? a.draft : a.target;
                const Stat one = stat_of(g, of.row(r, j), of.type, 0, a.n,
                                         side ? inverse_q : inverse_p);
                (side ? q : p) = one;
            }
            if (j == length)
                break;
            int how = decide(a, r, j, inverse_p, inverse_q, p, q, kLoose);
            if (how == kOpen)
                how = decide_exactly(g, a, r, j, inverse_p, inverse_q, p, q);
            if (how == kRejected)
                break;
        }
        int32_t token = -1;
        if (!is_masked(p, a.target.type)) {
            if (inverse_p > 0.0) {
                const Draw d = draw_of(a, r, j, length, inverse_p, inverse_q, p, q);
                token = settle(g, d, draw_part(g, d, 0, a.n));
            } else {
                token = p.first;
            }
        }
        if (g.t == 0)
            answer(a, r, j, token, inverse_p, p);
    }
}

// ---- long rows ----

__global__ __launch_bounds__(256) void k_verify_clear(VerifyArgs a)
{
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < a.n_requests;
         r += (int64_t)gridDim.x * 256) {
        a.rejected[r] = INT32_MAX;
        a.done[r] = 0;
    }
}

// The stats of row i of request r, target's and drafter's, or of a part of them.  Whole rows
// (WHOLE): rows i of all requests before rows i + 1 of any, and a row behind a draft that is
// known to be rejected by then is left out: nobody asks for it.
template <int G, bool WHOLE>
__global__ __launch_bounds__(G) void k_verify_rows(VerifyArgs a)
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
        if (!WHOLE && i == 0 && part == 0 && g.t == 0)
            a.done[r] = 0;
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
        Stat p, q = {0, 0, 0.0};
        const bool both = i < length && has_row(a, inverse_q) && inverse_p > 0.0;
        for (int side = 0; side <= (int)both; ++side) {
            const Side &of = side ? a.draft : a.target;
            const Stat one = stat_of(g, of.row(r, i), of.type, lo, hi,
                                     side ? inverse_q : inverse_p);
            (side ? q : p) = one;
        }
        if (g.t == 0) {
            a.stat(r, i, 0)[part] = p;
            a.stat(r, i, 1)[part] = q;
            if (WHOLE && i < length &&
                decide(a, r, i, inverse_p, inverse_q, p, q, kLoose) == kRejected)
                atomicMin(&a.rejected[r], i);
        }
    }
}

constexpr int kDrawBlock = 256;

__global__ __launch_bounds__(kDrawBlock) void k_verify_draw(VerifyArgs a)
{
    constexpr int G = kDrawBlock;
    __shared__ Scratch scratch;
    __shared__ uint32_t place;
    Group<G> g(threadIdx.x, &scratch);
    const int lane = threadIdx.x % kWave;
    const int64_t units = a.n_requests * a.draw_parts;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int64_t r = unit / a.draw_parts;
        const int32_t part = (int32_t)(unit - r * a.draw_parts);
        const double inverse_p = a.target.inverse_of(r), inverse_q = a.draft.inverse_of(r);
        const int32_t length = a.length(r);
        // the walk, 64 drafts at a time and the same in every wave of the block
        int32_t j = length;
        for (int32_t base = 0; base < length && j == length; base += kWave) {
            const int32_t i = base + lane;
            int how = kAccepted;
            Stat p = {0, 0, 0.0}, q = p;
            if (i < length) {
                p = join(a.stat(r, i, 0), a.parts, a.target.type, inverse_p);
                if (has_row(a, inverse_q) && inverse_p > 0.0)
                    q = join(a.stat(r, i, 1), a.parts, a.draft.type, inverse_q);
                how = decide(a, r, i, inverse_p, inverse_q, p, q, kLoose);
            }
            uint64_t ends = __ballot(how != kAccepted);
            while (ends) {
                const int k = __builtin_ctzll(ends);
                ends &= ends - 1;
                int one = __shfl(how, k);
                if (one == kOpen) {
                    Stat pk = {(uint32_t)__shfl((int)p.m, k), 0, 0.0}, qk = pk;
                    qk.m = (uint32_t)__shfl((int)q.m, k);
                    one = decide_exactly(g, a, r, base + k, inverse_p, inverse_q, pk, qk);
                }
                if (one == kRejected) {
                    j = base + k;
                    break;
                }
            }
        }
        const Stat p = join(a.stat(r, j, 0), a.parts, a.target.type, inverse_p);
        if (inverse_p == 0.0 || is_masked(p, a.target.type)) {
            if (part == 0 && g.t == 0)
                answer(a, r, j, is_masked(p, a.target.type) ? -1 : p.first, inverse_p, p);
            continue;
        }
        Stat q = {0, 0, 0.0};
        if (j < length && has_row(a, inverse_q))
            q = join(a.stat(r, j, 1), a.parts, a.draft.type, inverse_q);
        const Draw d = draw_of(a, r, j, length, inverse_p, inverse_q, p, q);
        const int32_t lo = part * a.draw_part;
        Best best = draw_part(g, d, lo, min(a.n, lo + a.draw_part));
        if (a.draw_parts > 1) {
            Best *of = a.bests + r * a.draw_parts;
            if (g.t == 0) {
                // past this die's caches, before the count says that it is there
                uint64_t w[4];
                __builtin_memcpy(w, &best, sizeof w);
                for (int k = 0; k < 4; ++k)
                    __hip_atomic_store(reinterpret_cast<uint64_t *>(of + part) + k, w[k],
                                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                place = __hip_atomic_fetch_add(&a.done[r], 1u, __ATOMIC_ACQ_REL,
                                               __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            const bool last = place == (uint32_t)a.draw_parts - 1;
            __syncthreads();
            if (!last)
                continue;
            best = nothing();
            for (int32_t k = g.t; k < a.draw_parts; k += G) {
                uint64_t w[4];
                for (int e = 0; e < 4; ++e)
                    w[e] = __hip_atomic_load(reinterpret_cast<uint64_t *>(of + k) + e,
                                             __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                Best one;
                __builtin_memcpy(&one, w, sizeof one);
                merge(best, one);
            }
            best = join(g, best);
        }
        const int32_t token = settle(g, d, best);
        if (g.t == 0)
            answer(a, r, j, token, inverse_p, p);
    }
}

// ---- which form, and its workspace ----
constexpr int32_t kShortClasses = 4096;
constexpr int kWholeBlock = 1024;

struct Plan {
    bool is_short, whole;
    int32_t parts, part, draw_parts, draw_part;
    size_t stats, rejected, done, bests, bytes;
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
    p.is_short = n <= kShortClasses;
    if (p.is_short || n_requests == 0)
        return p;
    const int64_t rows = n_requests * (drafts + 1);
    p.whole = rows >= 512;
    split(rows, n, p.whole ? 1 : 1024, 4096, p.parts, p.part);
    split(n_requests, n, 1024, 4096, p.draw_parts, p.draw_part);
    p.rejected = up((size_t)rows * 2 * p.parts * sizeof(Stat));
    p.done = p.rejected + up((size_t)n_requests * 4);
    p.bests = p.done + up((size_t)n_requests * 4);
    p.bytes = p.bests + (p.draw_parts > 1 ? (size_t)n_requests * p.draw_parts * sizeof(Best) : 0);
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
        hipLaunchKernelGGL(k_verify_short, grid((n_requests + kGroups - 1) / kGroups),
                           dim3(kShortBlock), 0, stream, a);
        return hipGetLastError();
    }
    char *ws = static_cast<char *>(workspace);
    a.stats = reinterpret_cast<Stat *>(ws);
    a.rejected = reinterpret_cast<int32_t *>(ws + p.rejected);
    a.done = reinterpret_cast<uint32_t *>(ws + p.done);
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
    return hipGetLastError();
}

}  // namespace bl
