// Kernels of low-rank adapters (internal), included once for each weight type W (float32,
// float16, bfloat16); x of type X, W or int32.
//
// A tile has up to 32 rows of one adapter.  out = base + scale up (down x) is two products on
// the matrix cores:
//
//   h [rank][rows]    = down [rank][k] x^T [k][rows]
//   out^T [m][rows]   = up [m][rank] h [rank][rows]
//
// With rows in the columns of both, a lane ends the first product with h at row l % 16 and
// ranks 4 (l / 16) + i, i < 4 (l its place in the wave), which is what it has to hand to the
// second, if the order of its terms is chosen so.  Narrow adapters are one kernel, a wave a
// tile, and h never leaves its registers.  Wide ones are two, k_shrink with the k terms dealt to
// waves and blocks and k_expand with the m columns, since a tile's waves alone are too few to
// keep memory busy (8192 rows, 4096 -> 4096, rank 64: 162 us in one kernel of 4 waves a tile);
// h goes through the workspace, a few bytes beside the row it is made of.
//
// 16-bit weights take h as the sum of two terms of their type, in the two halves of one
// instruction's terms: 2^-17 of h in bfloat16, 2^-22 of the row's largest in float16, whose
// rows of h are scaled by powers of two, since h may be past its range.  One term alone would
// round h to 2^-9 or 2^-12.
//
// Operands come from memory in the lanes' own layout, 16 bytes a load, without LDS: a row's
// 128 bytes by 8 loads of 16 lanes each.  Where a matrix lies the other way round (the
// gradient of x takes up^T and down^T), a lane loads 4 rows of 8 columns and picks its terms
// by byte permutes; its output columns are then 8 neighbours.
//
// What bounds it: memory; x, base and out once, an adapter once a tile (from the L2 but for
// the first).
#pragma once

#include "adapters.h"

namespace bl {
namespace adapt {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int T> constexpr int kSize = T == kF16 || T == kBf16 ? 2 : 4;
template <int T> constexpr int kEls = 16 / kSize<T>;      // elements of a 16-byte load

// 16 bytes of a matrix operand: kEls terms of one row (or column).
struct Frag {
    uint32_t w[4];
};

__device__ __forceinline__ f32x4 mma_f32(Frag a, Frag b, f32x4 c)
{
#pragma unroll
    for (int u = 0; u < 4; ++u)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w[u]),
                                                 __uint_as_float(b.w[u]), c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f32x4 mma_f16(Frag a, Frag b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma_bf16(Frag a, Frag b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Terms of the weights' type on both sides.
template <int W>
__device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c)
{
    if constexpr (W == kF32)
        return mma_f32(a, b, c);
    else if constexpr (W == kF16)
        return mma_f16(a, b, c);
    else
        return mma_bf16(a, b, c);
}

__device__ __forceinline__ uint32_t bf16_bits(float v)    // to the nearest, ties to even
{
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v);
}
__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// v as the sum of two bfloat16; an infinity stays one.
__device__ __forceinline__ void split(float v, uint32_t &hi, uint32_t &lo)
{
    hi = bf16_bits(v);
    const float rest = v - bf16_value(hi);
    lo = bf16_bits((hi & 0x7FFFu) == 0x7F80u ? 0.0f : rest);
}

// An element's bits from float, rounded to the nearest, ties to even.
template <int T>
__device__ __forceinline__ uint32_t el_bits(float v)
{
    if constexpr (T == kF16)
        return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v);
    else if constexpr (T == kBf16)
        return bf16_bits(v);
    else
        return __float_as_uint(v);
}

// kEls elements from p, of which `left` are there; the others are zero.
template <int T>
__device__ __forceinline__ Frag load_frag(const char *p, int left)
{
    Frag f;
    if (left >= kEls<T>) {
        __builtin_memcpy(f.w, p, 16);
        return f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        f.w[i] = 0;
#pragma unroll
    for (int u = 0; u < kEls<T>; ++u)
        if (u < left) {
            if constexpr (kSize<T> == 4)
                f.w[u] = reinterpret_cast<const uint32_t *>(p)[u];
            else
                f.w[u / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[u]
                              << (16 * (u & 1));
        }
    return f;
}

template <int X>
__device__ __forceinline__ Frag to_terms(Frag f)          // int32 terms as float32
{
    if constexpr (X == kI32)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f.w[i] = __float_as_uint((float)(int32_t)f.w[i]);
    return f;
}

// A tile's h as terms of the second product, by 4 ranks: in 16-bit types their two parts.
// factor: what the rows' sums are to be multiplied by for it.
template <int W, int RT, int CT>
__device__ __forceinline__ void make_terms(const f32x4 (&h)[RT][CT], Frag (&terms)[RT][CT],
                                           float (&factor)[RT])
{
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        factor[rt] = 1.0f;
        float up = 1.0f;
        if constexpr (W == kF16) {
            // the row's largest to [2^8, 2^9): parts of it down to 2^-24 remain
            float most = 0.0f;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    most = fmaxf(most, fabsf(h[rt][ct][i]));
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            const int power = min(max(262 - (int)(__float_as_uint(most) >> 23), 1), 253);
            up = __uint_as_float((uint32_t)power << 23);
            factor[rt] = __uint_as_float((uint32_t)(254 - power) << 23);
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            Frag &f = terms[rt][ct];
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (W == kF32) {
                    f.w[i] = __float_as_uint(h[rt][ct][i]);
                } else if constexpr (W == kBf16) {
                    split(h[rt][ct][i], hi[i], lo[i]);
                } else {
                    const float v = h[rt][ct][i] * up;
                    const _Float16 part = (_Float16)v;
                    const float rest = v - (float)part;
                    hi[i] = __builtin_bit_cast(uint16_t, part);
                    lo[i] = __builtin_bit_cast(uint16_t, (_Float16)((hi[i] & 0x7FFFu) == 0x7C00u
                                                                        ? 0.0f : rest));
                }
            }
            if constexpr (W != kF32) {
                f.w[0] = hi[0] | hi[1] << 16;
                f.w[1] = hi[2] | hi[3] << 16;
                f.w[2] = lo[0] | lo[1] << 16;
                f.w[3] = lo[2] | lo[3] << 16;
            }
        }
    }
}

// c += w h for 4 ranks of w (two words of 16-bit weights, four of float32).
template <int W>
__device__ __forceinline__ f32x4 mma_h(const uint32_t (&w)[kSize<W>], Frag h, f32x4 c)
{
    if constexpr (W == kF32)
        return mma_f32({w[0], w[1], w[2], w[3]}, h, c);
    else
        return mma<W>({w[0], w[1], w[0], w[1]}, h, c);
}

// base and out of one row: out columns [col, col + kEls) from their sums, as many as there are.
template <int W>
struct Output {
    const char *base;                   // the row's, or NULL
    char *out;
    bool base_i32, there;
    float base_scale, scale;
    int32_t m;

    __device__ __forceinline__ void store(int32_t col, bool whole, const float (&sum)[kEls<W>],
                                          const Frag &b) const
    {
        if (!there)
            return;
        uint32_t bits[kEls<W>];
#pragma unroll
        for (int u = 0; u < kEls<W>; ++u) {
            float v = scale * sum[u];
            if (base) {
                float from;
                if constexpr (W == kF32)
                    from = base_i32 ? (float)(int32_t)b.w[u] : __uint_as_float(b.w[u]);
                else if constexpr (W == kBf16)
                    from = __uint_as_float(u & 1 ? b.w[u / 2] & 0xFFFF0000u : b.w[u / 2] << 16);
                else
                    from = (float)__builtin_bit_cast(_Float16,
                                                     (uint16_t)(b.w[u / 2] >> (16 * (u & 1))));
                v += base_scale * from;
            }
            bits[u] = el_bits<W>(v);
        }
        char *to = out + (int64_t)col * kSize<W>;
        if (whole) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = kSize<W> == 4 ? bits[i] : bits[2 * i] | bits[2 * i + 1] << 16;
            __builtin_memcpy(to, w, 16);
        } else {
#pragma unroll
            for (int u = 0; u < kEls<W>; ++u)
                if (col + u < m) {
                    if constexpr (kSize<W> == 4)
                        reinterpret_cast<uint32_t *>(to)[u] = bits[u];
                    else
                        reinterpret_cast<uint16_t *>(to)[u] = (uint16_t)bits[u];
                }
        }
    }
};

// A tile and the lane's rows in it: 16 rt + l % 16.
template <int RT>
struct Tile {
    Piece4 p;
    int32_t row[RT];
    bool there[RT];

    // false: no tile
    __device__ __forceinline__ bool take(const PassArgs &a, int64_t tile, int col)
    {
        if (a.tiles) {
            p = a.tiles[tile];
            if (p.group < 0)
                return false;
        } else {
            const int32_t id = a.ids[tile];
            p = {id >= 0 && id < a.groups ? id : a.groups, (int32_t)tile, 1, 0};
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int32_t at = rt * 16 + col;
            there[rt] = at < p.count;
            const int32_t place = p.first + (there[rt] ? at : 0);
            row[rt] = a.order ? a.order[place] : place;
        }
        return true;
    }
};

// Which of the E terms from k on a lane takes at the end of a row of n: it loads the row's last
// E instead, which start `back` terms earlier, and keeps those that are its own.
template <int W>
struct End {
    int32_t at;                         // where it loads
    uint32_t keep[4];                   // of the words there

    __device__ __forceinline__ End(int32_t k, int32_t n)
    {
        constexpr int E = kEls<W>;
        at = min(k, n - E);
        const int32_t back = k - at;    // (E or more: none is its own)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (kSize<W> == 4)
                keep[i] = i >= back ? 0xFFFFFFFFu : 0u;
            else
                keep[i] = (2 * i >= back ? 0x0000FFFFu : 0u) |
                          (2 * i + 1 >= back ? 0xFFFF0000u : 0u);
        }
    }
    __device__ __forceinline__ Frag take(Frag f) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f.w[i] &= keep[i];
        return f;
    }
};

__device__ __forceinline__ Frag load_16(const char *p)
{
    Frag f;
    __builtin_memcpy(f.w, p, 16);
    return f;
}

// E terms of a column of a matrix with `step` bytes from term to term.
template <int W>
__device__ __forceinline__ Frag load_across(const char *p, int64_t step)
{
    Frag f;
    if constexpr (kSize<W> == 4) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            f.w[u] = *reinterpret_cast<const uint32_t *>(p + u * step);
    } else {
        uint32_t v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            v[u] = *reinterpret_cast<const uint16_t *>(p + u * step);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f.w[i] = v[2 * i] | v[2 * i + 1] << 16;
    }
    return f;
}

// h += w1 x over terms [from, to): units of 128 bytes of a row, every `deal`-th from the
// `turn`-th on; `to` is k or a multiple of the unit.  A unit's loads are issued before the
// products of the one before.
template <int W, int X, int CT, int RT, bool BACK>
__device__ __forceinline__ void shrink(const PassArgs &a, const Tile<RT> &tile, int col, int quad,
                                       int32_t from, int32_t to, int turn, int deal,
                                       f32x4 (&h)[RT][CT])
{
    constexpr int E = kEls<W>, S = kSize<W>, kUnit = 8 * E;
    const char *x[RT], *w1[CT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
        x[rt] = a.x + tile.row[rt] * a.x_stride;
    const char *first = a.w1 + tile.p.group * a.w1_step;
    const int64_t across = (int64_t)a.rank * S;           // BACK: from term to term
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        // ranks behind the last one read its weights: what comes of it is cleared afterwards
        const int32_t r = min(ct * 16 + col, a.rank - 1);
        w1[ct] = first + (BACK ? (int64_t)r : (int64_t)r * a.k) * S;
    }
    struct Unit {
        Frag x[2][RT], w[2][CT];
    };
    const auto load = [&](Unit &u, int32_t k0) __attribute__((always_inline)) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int32_t k = k0 + half * 4 * E + quad * E;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                u.x[half][rt] = load_16(x[rt] + (int64_t)k * S);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
                u.w[half][ct] = BACK ? load_across<W>(w1[ct] + k * across, across)
                                     : load_16(w1[ct] + (int64_t)k * S);
        }
    };
    const auto products = [&](const Unit &u) __attribute__((always_inline)) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const Frag t = to_terms<X>(u.x[half][rt]);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
                    h[rt][ct] = mma<W>(u.w[half][ct], t, h[rt][ct]);
            }
    };
    const int32_t whole = min(to, a.k / kUnit * kUnit), step = deal * kUnit;
    int32_t k0 = from + turn * kUnit;
    if (k0 < whole) {
        Unit now, next;
        load(now, k0);
        for (;;) {
            k0 += step;
            if (k0 >= whole)
                break;
            load(next, k0);
            products(now);
            now = next;
        }
        products(now);
    }
    if (k0 < to) {                                        // the row's last terms
        Unit u;
        if (a.k >= E) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const End<W> end(k0 + half * 4 * E + quad * E, a.k);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    u.x[half][rt] = end.take(load_16(x[rt] + (int64_t)end.at * S));
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
                    u.w[half][ct] = end.take(
                        BACK ? load_across<W>(w1[ct] + end.at * across, across)
                             : load_16(w1[ct] + (int64_t)end.at * S));
            }
        } else {                                          // fewer than one load's
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int32_t left = half == 0 && quad == 0 ? a.k : 0;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    u.x[half][rt] = load_frag<W>(x[rt], left);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    Frag f = {{0, 0, 0, 0}};
                    for (int32_t i = 0; i < left; ++i) {  // (a run-time index of few)
                        const char *el = w1[ct] + i * (BACK ? across : S);
                        const uint32_t v = S == 4 ? *reinterpret_cast<const uint32_t *>(el)
                                                  : *reinterpret_cast<const uint16_t *>(el);
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (e == i)
                                f.w[e * S / 4] |= S == 4 ? v : v << (16 * (e & 1));
                    }
                    u.w[half][ct] = f;
                }
            }
        }
        products(u);
    }
}

template <int RT, int CT>
__device__ __forceinline__ void clear(f32x4 (&h)[RT][CT])
{
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
            h[rt][ct] = f32x4{0, 0, 0, 0};
}

template <int RT, int CT>
__device__ __forceinline__ void clear_past_rank(int32_t rank, int quad, f32x4 (&h)[RT][CT])
{
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (ct * 16 + quad * 4 + i >= rank)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    h[rt][ct][i] = 0.0f;
}

template <int RT, int CT>
__device__ __forceinline__ void store_hidden(float *to, int32_t rank, const Tile<RT> &tile,
                                             int quad, const f32x4 (&h)[RT][CT])
{
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
        if (tile.there[rt])
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const int32_t r = ct * 16 + quad * 4;
                float *at = to + (int64_t)tile.row[rt] * rank + r;
                if (r + 4 <= rank) {
                    __builtin_memcpy(at, &h[rt][ct], 16);
                } else {
#pragma unroll
                    for (int i = 0; i < 3; ++i)
                        if (r + i < rank)
                            at[i] = h[rt][ct][i];
                }
            }
}

// Four ranks of a row of `rank` from r on; zeros past the last one.
template <int W>
__device__ __forceinline__ void load_ranks(const char *row, int32_t r, int32_t rank,
                                           uint32_t (&w)[kSize<W>])
{
    constexpr int S = kSize<W>;
    if (r + 4 <= rank) {
        __builtin_memcpy(w, row + r * S, 4 * S);
        return;
    }
#pragma unroll
    for (int i = 0; i < S; ++i)
        w[i] = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (r + i < rank) {
            if constexpr (S == 4)
                w[i] = reinterpret_cast<const uint32_t *>(row)[r + i];
            else
                w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[r + i]
                            << (16 * (i & 1));
        }
}

// out = base + scale w2 h: units of columns, every `deal`-th from the `turn`-th on.  The next
// unit's base is loaded, and the next weights where registers allow, before this one's products.
template <int W, int CT, int RT, bool BACK>
struct Expand {
    static constexpr int E = kEls<W>, S = kSize<W>;
    static constexpr int kCols = BACK ? 16 * E : 32;      // of a unit
    static constexpr int kPieces = S == 2 ? 1 : 2;        // forward: loads of base a row
    static constexpr bool kAhead = (BACK ? 16 : 2 * S) * CT <= 32;
    struct Weights {
        uint32_t w[BACK ? 1 : 2][CT][S];                  // forward: 4 ranks of two tiles' rows
        Frag f[BACK ? CT : 1][4];                         // back: 4 ranks of E columns
    };
    struct Base {
        Frag f[RT][kPieces];
    };
    const PassArgs &a;
    const char *w2;
    Output<W> o[RT];
    int col, quad;
    bool adapted;

    __device__ __forceinline__ Expand(const PassArgs &args, const Tile<RT> &tile, int c, int q)
        : a(args), col(c), quad(q), adapted(tile.p.group < args.groups)
    {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            o[rt].base = BACK || !a.base ? nullptr : a.base + tile.row[rt] * a.base_stride;
            o[rt].out = a.out + tile.row[rt] * a.out_stride;
            o[rt].base_i32 = a.base_i32;
            o[rt].there = tile.there[rt];
            o[rt].base_scale = a.base_scale;
            o[rt].m = a.m;
            o[rt].scale = !adapted ? 0.0f : a.scales ? a.scales[tile.p.group] : a.scale;
        }
        w2 = a.w2 + (adapted ? tile.p.group * a.w2_step : 0);
    }
    __device__ __forceinline__ void load_base(Base &b, int32_t m0) const
    {
        if constexpr (!BACK) {
            if (!a.base)
                return;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int32_t m = m0 + i * 16 + quad * E;
                    if (m0 + kCols <= a.m)                // (rows that are not there: the first)
                        b.f[rt][i] = load_16(o[rt].base + (int64_t)m * S);
                    else
                        b.f[rt][i] = load_frag<W>(o[rt].base + (int64_t)m * S, a.m - m);
                }
        }
    }
    // forward: the tiles' rows of w2; 16-bit types give a lane 8 neighbours of them
    __device__ __forceinline__ int32_t column(int t) const
    {
        return S == 2 ? col / 4 * 8 + t * 4 + col % 4 : t * 16 + col;
    }
    __device__ __forceinline__ void load_weights(Weights &w, int32_t m0) const
    {
        if (!adapted)
            return;
        if constexpr (!BACK) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const char *row = w2 + (int64_t)min(m0 + column(t), a.m - 1) * a.rank * S;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
                    load_ranks<W>(row, ct * 16 + quad * 4, a.rank, w.w[t][ct]);
            }
        } else {
            const int32_t m = m0 + col * E;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t r = ct * 16 + quad * 4 + i;
                    const char *from = w2 + ((int64_t)min(r, a.rank - 1) * a.m + m) * S;
                    Frag f;
                    if (m0 + kCols <= a.m)
                        f = load_16(from);
                    else
                        f = load_frag<W>(from, a.m - m);
#pragma unroll
                    for (int e = 0; e < 4; ++e)           // (their h is zero, they may be NaNs)
                        f.w[e] = r < a.rank ? f.w[e] : 0;
                    w.f[ct][i] = f;
                }
        }
    }
    __device__ __forceinline__ void unit(int32_t m0, const Weights &w, const Base &b,
                                         const Frag (&terms)[RT][CT]) const
    {
        constexpr int T = BACK ? E : 2;
        f32x4 sum[T][RT];
        clear(sum);
        if (adapted)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    uint32_t v[S];
                    if constexpr (!BACK) {
#pragma unroll
                        for (int i = 0; i < S; ++i)
                            v[i] = w.w[t][ct][i];
                    } else if constexpr (S == 4) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[i] = w.f[ct][i].w[t];
                    } else {
                        const uint32_t pick = t & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            v[i] = __builtin_amdgcn_perm(w.f[ct][2 * i + 1].w[t / 2],
                                                         w.f[ct][2 * i].w[t / 2], pick);
                    }
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
                        sum[t][rt] = mma_h<W>(v, terms[rt][ct], sum[t][rt]);
                }
        const bool whole = m0 + kCols <= a.m;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if constexpr (!BACK) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    float v[E];
#pragma unroll
                    for (int u = 0; u < E; ++u)
                        v[u] = sum[S == 2 ? u / 4 : i][rt][u % 4];
                    o[rt].store(m0 + i * 16 + quad * E, whole, v, b.f[rt][i]);
                }
            } else {
                // tile t has columns t, E + t, 2 E + t, ...
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[E];
#pragma unroll
                    for (int t = 0; t < E; ++t)
                        v[t] = sum[t][rt][i];
                    o[rt].store(m0 + (quad * 4 + i) * E, whole, v, {{0, 0, 0, 0}});
                }
            }
        }
    }
    __device__ __forceinline__ void run(int turn, int deal, Base &b, const f32x4 (&h)[RT][CT])
    {
        Weights w;
        int32_t m0 = turn * kCols;
        if (m0 >= a.m)
            return;
        if constexpr (kAhead)
            load_weights(w, m0);
        Frag terms[RT][CT];
        float factor[RT];
        make_terms<W>(h, terms, factor);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
            o[rt].scale *= factor[rt];
        for (;;) {
            const int32_t next = m0 + deal * kCols;
            Weights w_next;
            Base b_next;
            if constexpr (!kAhead)
                load_weights(w, m0);
            if (next < a.m) {
                load_base(b_next, next);
                if constexpr (kAhead)
                    load_weights(w_next, next);
            }
            unit(m0, w, b, terms);
            if (next >= a.m)
                return;
            m0 = next;
            b = b_next;
            if constexpr (kAhead)
                w = w_next;
        }
    }
};

// ---- narrow adapters: a wave a tile ----
template <int W, int X, int CT, bool BACK>
__global__ __launch_bounds__(256) void k_narrow(PassArgs a)
{
    constexpr int RT = kTile / 16;
    const int lane = threadIdx.x % kWave, col = lane % 16, quad = lane / 16;
    const int64_t at = (int64_t)blockIdx.x * 4 +
                       __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    Tile<RT> tile;
    if (at >= a.n_tiles || !tile.take(a, at, col))
        return;
    f32x4 h[RT][CT];
    clear(h);
    Expand<W, CT, RT, BACK> expand(a, tile, col, quad);
    typename Expand<W, CT, RT, BACK>::Base b;
    if (a.out)
        expand.load_base(b, 0);
    if (tile.p.group < a.groups) {
        shrink<W, X, CT, RT, BACK>(a, tile, col, quad, 0, a.k, 0, 1, h);
        clear_past_rank(a.rank, quad, h);
    }
    if (a.hidden)
        store_hidden(a.hidden, a.rank, tile, quad, h);
    if (a.out)
        expand.run(0, 1, b, h);
}

// ---- wide adapters ----
constexpr int kWideWaves = 4;
// waves that share a block's terms: as many as a rank's sums leave LDS for
template <int CT> constexpr int kTermWaves = CT <= 2 ? 8 : 4;

// Part `blockIdx % splits` of a tile's h, to [part][row][rank].
template <int W, int X, int CT, int RT, bool BACK>
__global__ __launch_bounds__(kTermWaves<CT> * kWave) void k_shrink(PassArgs a)
{
    constexpr int NW = kTermWaves<CT>, kAcc = CT * RT * 4, kUnit = 8 * kEls<W>;
    __shared__ float joined[NW * kAcc * kWave];
    const int lane = threadIdx.x % kWave, col = lane % 16, quad = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int64_t at = blockIdx.x / a.splits;
    const int part = (int)(blockIdx.x - at * a.splits);
    Tile<RT> tile;
    if (!tile.take(a, at, col))
        return;
    f32x4 h[RT][CT];
    clear(h);
    if (tile.p.group < a.groups) {
        const int32_t units = (a.k + kUnit - 1) / kUnit;
        const int32_t each = (units + a.splits - 1) / a.splits;
        const int32_t from = min(part * each, units) * kUnit;
        const int32_t to = min(min((part + 1) * each, units) * kUnit, a.k);
        shrink<W, X, CT, RT, BACK>(a, tile, col, quad, from, to, wave, NW, h);
        clear_past_rank(a.rank, quad, h);
        // the waves' sums, added in order; each wave adds up some of them
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    joined[(wave * kAcc + (rt * CT + ct) * 4 + i) * kWave + lane] = h[rt][ct][i];
        __syncthreads();
    }
    // wave w stores fragments w, w + NW, ... of the tile's RT * CT
#pragma unroll
    for (int f = 0; f < RT * CT; ++f) {
        if (f % NW != wave)
            continue;
        f32x4 sum = {0, 0, 0, 0};
        if (tile.p.group < a.groups)
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sum[i] += joined[(w * kAcc + f * 4 + i) * kWave + lane];
        const int rt = f / CT, r = f % CT * 16 + quad * 4;
        if (!tile.there[rt] || r >= a.rank)
            continue;
        float *to = a.partial + ((int64_t)part * a.n_rows + tile.row[rt]) * a.rank + r;
        if (r + 4 <= a.rank) {
            __builtin_memcpy(to, &sum, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (r + i < a.rank)
                    to[i] = sum[i];
        }
    }
}

template <int W, int CT, int RT, bool BACK>
__global__ __launch_bounds__(kWideWaves * kWave) void k_expand(PassArgs a, int32_t blocks)
{
    const int lane = threadIdx.x % kWave, col = lane % 16, quad = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int64_t at = blockIdx.x / blocks;
    const int block = (int)(blockIdx.x - at * blocks);
    Tile<RT> tile;
    if (!tile.take(a, at, col))
        return;
    Expand<W, CT, RT, BACK> expand(a, tile, col, quad);
    typename Expand<W, CT, RT, BACK>::Base b;
    const int turn = block * kWideWaves + wave;
    if (a.out && turn * expand.kCols < a.m)
        expand.load_base(b, turn * expand.kCols);
    f32x4 h[RT][CT];
    clear(h);
#pragma unroll(CT <= 2 ? 2 : 1)
    for (int32_t p = 0; p < a.splits; ++p)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float *from = a.partial + (p * a.n_rows + tile.row[rt]) * a.rank;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                uint32_t w[4];
                load_ranks<kF32>(reinterpret_cast<const char *>(from), ct * 16 + quad * 4, a.rank,
                                 w);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    h[rt][ct][i] += __uint_as_float(w[i]);
            }
        }
    if (a.hidden && a.hidden != a.partial && block == 0 && wave == 0)
        store_hidden(a.hidden, a.rank, tile, quad, h);
    if (a.out)
        expand.run(turn, blocks * kWideWaves, b, h);
}

template <int W, int X, int CT, bool BACK>
hipError_t pass_of(const PassArgs &a, hipStream_t stream)
{
    if (a.splits == 0) {
        hipLaunchKernelGGL((k_narrow<W, X, CT, BACK>), dim3((uint32_t)((a.n_tiles + 3) / 4)),
                           dim3(256), 0, stream, a);
        return hipGetLastError();
    }
    const dim3 parts((uint32_t)(a.n_tiles * a.splits)), term_waves(kTermWaves<CT> * kWave);
    if (a.tiles)
        hipLaunchKernelGGL((k_shrink<W, X, CT, 2, BACK>), parts, term_waves, 0, stream, a);
    else
        hipLaunchKernelGGL((k_shrink<W, X, CT, 1, BACK>), parts, term_waves, 0, stream, a);
    if (hipError_t err = hipGetLastError(); err != hipSuccess)
        return err;
    if (!a.out && a.hidden == a.partial)
        return hipSuccess;
    // about 2048 blocks, of 512 columns at most and a unit a wave at least
    constexpr int kLeast = kWideWaves * Expand<W, CT, 2, BACK>::kCols;
    const int64_t least = (a.m + kLeast - 1) / kLeast, most = (a.m + 511) / 512;
    const int32_t blocks = !a.out ? 1 : (int32_t)std::min<int64_t>(
        least, std::max<int64_t>(most, 2048 / a.n_tiles));
    const dim3 grid((uint32_t)(a.n_tiles * blocks)), waves(kWideWaves * kWave);
    if (a.tiles)
        hipLaunchKernelGGL((k_expand<W, CT, 2, BACK>), grid, waves, 0, stream, a, blocks);
    else
        hipLaunchKernelGGL((k_expand<W, CT, 1, BACK>), grid, waves, 0, stream, a, blocks);
    return hipGetLastError();
}

template <int W, int X, bool BACK>
hipError_t pass_by_rank(const PassArgs &a, hipStream_t stream)
{
    if (a.rank <= 16)
        return pass_of<W, X, 1, BACK>(a, stream);
    if (a.rank <= 32)
        return pass_of<W, X, 2, BACK>(a, stream);
    if (a.rank <= 64)
        return pass_of<W, X, 4, BACK>(a, stream);
    return pass_of<W, X, 8, BACK>(a, stream);
}

// ---- gradients of the weights ----
// D [rank][cols] = sum over a chunk's rows of h[row][rank] y[row][col]: a block has 16 E
// columns, and its waves share the rows, 32 (16 in float32) a step; a lane loads E columns of
// 8 (4) rows and turns them by byte permutes into the terms of E products, whose columns are
// t, E + t, ...  h is taken as the sum of two bfloat16 as above, float16 y too, since h may be
// past float16's range and its rows are summed here, so that they have no scale of their own.
constexpr int kGradWaves = 4;

template <int W, int CT>
__global__ __launch_bounds__(kGradWaves * kWave) void k_grads(GradArgs a)
{
    constexpr int E = kEls<W>, S = kSize<W>, kRows = S == 4 ? 4 : 8;   // rows a lane and step
    constexpr int NW = kGradWaves, kStep = 4 * kRows;
    __shared__ float joined[NW * E * 4 * kWave];
    const int lane = threadIdx.x % kWave, col = lane % 16, quad = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int32_t blocks = a.job[0].blocks + a.job[1].blocks;
    const int64_t chunk = blockIdx.x / blocks;
    int32_t block = (int32_t)(blockIdx.x - chunk * blocks);
    const bool second = block >= a.job[0].blocks;
    const GradJob &j = a.job[second];
    block -= second ? a.job[0].blocks : 0;
    const Piece4 p = a.chunks[chunk];
    if (p.group < 0 || p.group >= a.groups)
        return;
    const int32_t c0 = block * 16 * E, at = c0 + col * E, left = max(j.cols - at, 0);
    const bool whole_block = c0 + 16 * E <= j.cols;
    f32x4 sum[CT][E];
    clear(sum);
    const char *y = j.y + (left > 0 ? (int64_t)at * S : 0);
    const int32_t *order = a.order + p.first;
    for (int32_t s = wave * kStep; s < p.count; s += NW * kStep) {
        const bool whole_step = s + kStep <= p.count;
        Frag f[kRows];
        float hv[CT][kRows];
        int32_t row[kRows];
        if (whole_step) {
            __builtin_memcpy(row, order + s + quad * kRows, sizeof row);
        } else {
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                row[u] = order[min(s + quad * kRows + u, p.count - 1)];
        }
        if (whole_block) {
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                __builtin_memcpy(f[u].w, y + row[u] * j.y_stride, 16);
        } else {
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                f[u] = load_frag<W>(y + row[u] * j.y_stride, left);
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int32_t r = min(ct * 16 + col, a.rank - 1);   // (past the rank: not stored)
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                hv[ct][u] = j.h[(int64_t)row[u] * a.rank + r];
        }
        if (!whole_step)                                  // rows past the chunk's last
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                if (s + quad * kRows + u >= p.count) {
                    f[u] = {{0, 0, 0, 0}};
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
                        hv[ct][u] = 0.0f;
                }
        if constexpr (S == 4) {
            if (j.y_i32)
#pragma unroll
                for (int u = 0; u < kRows; ++u)
                    f[u] = to_terms<kI32>(f[u]);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const Frag hf = {{__float_as_uint(hv[ct][0]), __float_as_uint(hv[ct][1]),
                                  __float_as_uint(hv[ct][2]), __float_as_uint(hv[ct][3])}};
#pragma unroll
                for (int t = 0; t < E; ++t)
                    sum[ct][t] = mma_f32(hf, {{f[0].w[t], f[1].w[t], f[2].w[t], f[3].w[t]}},
                                         sum[ct][t]);
            }
        } else {
            Frag hi[CT], lo[CT];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t h0, l0, h1, l1;
                    split(hv[ct][2 * i], h0, l0);
                    split(hv[ct][2 * i + 1], h1, l1);
                    hi[ct].w[i] = h0 | h1 << 16;
                    lo[ct].w[i] = l0 | l1 << 16;
                }
#pragma unroll
            for (int t = 0; t < E; ++t) {
                const uint32_t pick = t & 1 ? 0x07060302u : 0x05040100u;
                Frag b;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    b.w[i] = __builtin_amdgcn_perm(f[2 * i + 1].w[t / 2], f[2 * i].w[t / 2],
                                                   pick);
                Frag rest;
                if constexpr (W == kF16)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t h0, l0, h1, l1;
                        split((float)__builtin_bit_cast(_Float16, (uint16_t)b.w[i]), h0, l0);
                        split((float)__builtin_bit_cast(_Float16, (uint16_t)(b.w[i] >> 16)), h1,
                              l1);
                        b.w[i] = h0 | h1 << 16;
                        rest.w[i] = l0 | l1 << 16;
                    }
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    sum[ct][t] = mma_bf16(hi[ct], b, sum[ct][t]);
                    sum[ct][t] = mma_bf16(lo[ct], b, sum[ct][t]);
                    if constexpr (W == kF16)
                        sum[ct][t] = mma_bf16(hi[ct], rest, sum[ct][t]);
                }
            }
        }
    }
    // The waves' sums, added in order, 16 ranks at a time; wave w has ranks 4 quad + w of them.
    // A group of one chunk is done, others leave a part of the sum.
    static_assert(NW == 4, "a wave an i");
    const bool done = a.chunk_starts[p.group + 1] - a.chunk_starts[p.group] == 1;
    const float scale = a.scales ? a.scales[p.group] : a.scale;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        if (ct > 0)
            __syncthreads();
#pragma unroll
        for (int t = 0; t < E; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                joined[((i * NW + wave) * E + t) * kWave + lane] = sum[ct][t][i];
        __syncthreads();
        const int32_t r = ct * 16 + quad * 4 + wave;
        float v[E];
#pragma unroll
        for (int t = 0; t < E; ++t) {
            v[t] = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w)
                v[t] += joined[((wave * NW + w) * E + t) * kWave + lane];
        }
        if (r >= a.rank)
            continue;
        if (!done) {
            float *to = j.partial + ((int64_t)p.slot * a.rank + r) * j.cols + at;
#pragma unroll
            for (int t = 0; t < E; ++t)
                if (t < left)
                    to[t] = v[t];
        } else {
            const int64_t base = (int64_t)p.group * a.rank * j.cols;
#pragma unroll
            for (int t = 0; t < E; ++t) {
                const int64_t to = base + (j.transposed ? (int64_t)(at + t) * a.rank + r
                                                        : (int64_t)r * j.cols + at + t);
                if (t < left) {
                    if constexpr (S == 4)
                        reinterpret_cast<uint32_t *>(j.out)[to] = el_bits<W>(scale * v[t]);
                    else
                        reinterpret_cast<uint16_t *>(j.out)[to] =
                            (uint16_t)el_bits<W>(scale * v[t]);
                }
            }
        }
    }
}

// Gradients of groups with no rows (zero) and of those with several chunks, whose parts are
// added in order.
template <int W>
__global__ __launch_bounds__(256) void k_join_grads(GradArgs a, int32_t per_group)
{
    const int32_t g = (int32_t)(blockIdx.x / per_group);
    if (a.chunk_starts && a.chunk_starts[g + 1] - a.chunk_starts[g] == 1)
        return;
    const int32_t first = a.chunk_starts ? a.slot_starts[g] : 0,
                  last = a.chunk_starts ? a.slot_starts[g + 1] : 0;
    const float scale = a.scales ? a.scales[g] : a.scale;
    for (int k = 0; k < 2; ++k) {
        const GradJob &j = a.job[k];
        if (!j.out)
            continue;
        const int64_t all = (int64_t)a.rank * j.cols;
        for (int64_t e = (int64_t)(blockIdx.x - g * per_group) * 256 + threadIdx.x; e < all;
             e += (int64_t)per_group * 256) {
            float v = 0.0f;
#pragma unroll 8
            for (int32_t c = first; c < last; ++c)
                v += j.partial[c * all + e];
            const int64_t r = e / j.cols, at = e - r * j.cols;
            const int64_t to = g * all + (j.transposed ? at * a.rank + r : e);
            if constexpr (kSize<W> == 4)
                reinterpret_cast<uint32_t *>(j.out)[to] = el_bits<W>(scale * v);
            else
                reinterpret_cast<uint16_t *>(j.out)[to] = (uint16_t)el_bits<W>(scale * v);
        }
    }
}

template <int W, int CT>
hipError_t grads_of(const GradArgs &a, hipStream_t stream)
{
    const int64_t blocks = a.n_chunks * (a.job[0].blocks + a.job[1].blocks);
    if (blocks > 0) {
        hipLaunchKernelGGL((k_grads<W, CT>), dim3((uint32_t)blocks), dim3(256), 0, stream, a);
        if (hipError_t err = hipGetLastError(); err != hipSuccess)
            return err;
    }
    const int64_t els = (int64_t)a.rank * std::max(a.job[0].out ? a.job[0].cols : 0,
                                                   a.job[1].out ? a.job[1].cols : 0);
    const int32_t per_group = (int32_t)std::min<int64_t>(1024, (els + 255) / 256);
    hipLaunchKernelGGL(k_join_grads<W>, dim3((uint32_t)((int64_t)a.groups * per_group)),
                       dim3(256), 0, stream, a, per_group);
    return hipGetLastError();
}

}  // namespace

template <int W>
hipError_t launch_pass(const PassArgs &a, bool x_i32, bool back, hipStream_t stream)
{
    if (back)
        return pass_by_rank<W, W, true>(a, stream);
    if constexpr (W == kF32)
        if (x_i32)
            return pass_by_rank<W, kI32, false>(a, stream);
    return pass_by_rank<W, W, false>(a, stream);
}

template <int W>
int32_t grad_block()
{
    return 16 * kEls<W>;
}

template <int W>
hipError_t launch_grads(const GradArgs &a, hipStream_t stream)
{
    if (a.rank <= 16)
        return grads_of<W, 1>(a, stream);
    if (a.rank <= 32)
        return grads_of<W, 2>(a, stream);
    if (a.rank <= 64)
        return grads_of<W, 4>(a, stream);
    return grads_of<W, 8>(a, stream);
}

}  // namespace adapt
}  // namespace bl
