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
// Memory is read and written by 8 lanes to 128 bytes of a row, which is where the matrix cores'
// layouts (16 lanes, 16 rows) touch four times the cache lines a byte: with those, the L1's tags
// were busy all the time (12289 x 5003 bfloat16 beside rank 24: 7.3e7 accesses, 1.1 a clock and
// CU, 109 us for 246 MB).  A wave turns its pieces in LDS of its own, without barriers; 16-byte
// slots are swizzled by the row.  A matrix whose rows are the ranks of one term (up, and
// its transpose in the gradient) is contiguous over a unit of terms and is copied as it lies.
// Where the gradient of x takes down^T, a lane loads 4 rows of 8 columns and picks its terms by
// byte permutes; its output columns are then 8 neighbours.
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

// kEls elements from p, of which `left` are there; the others are zero.  p is in a row of n
// elements that ends with them: if those are enough, its last ones are loaded and moved down.
// (An element at a time, each lane's loads are waited for one by one: the last block of 5003
// columns kept the gradients of 12289 rows waiting, 57 us for 48.)
template <int T>
__device__ __forceinline__ Frag load_frag(const char *p, int left, int64_t n)
{
    constexpr int E = kEls<T>, S = kSize<T>;
    Frag f;
    if (n >= E) {
        const int past = max(E - left, 0);
        __builtin_memcpy(f.w, p - (int64_t)past * S, 16);
        if (past > 0) {
            const int words = past * S / 4;
#pragma unroll
            for (int step = 1; step <= 4; step *= 2)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    f.w[i] = words >= 4 ? 0 : words & step ? (i + step < 4 ? f.w[i + step] : 0)
                                                           : f.w[i];
            if (S == 2 && (past & 1))
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    f.w[i] = f.w[i] >> 16 | (i < 3 ? f.w[i + 1] << 16 : 0);
        }
        return f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        f.w[i] = 0;
#pragma unroll
    for (int u = 0; u < E; ++u)
        if (u < left) {
            if constexpr (S == 4)
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

// ---- a wave's LDS ----
// Rows of 128 bytes in 16-byte slots; slot p of row r is at place p ^ (r % 8).
__device__ __forceinline__ int slot_at(int row, int p) { return row * 128 + ((p ^ (row & 7)) * 16); }

__device__ __forceinline__ Frag load_16(const char *p)
{
    Frag f;
    __builtin_memcpy(f.w, p, 16);
    return f;
}
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ Frag load_nt(const char *p)
{
    return __builtin_bit_cast(Frag, __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2 *>(p)));
}
__device__ __forceinline__ Frag lds_frag(const char *p) { return *reinterpret_cast<const Frag *>(p); }
__device__ __forceinline__ void lds_put(char *p, Frag f) { *reinterpret_cast<Frag *>(p) = f; }

// A tile, the wave's place in it, and the lane's rows: 8 j + l / 8.
template <int RT>
struct Tile {
    static constexpr int J = 2 * RT;
    Piece4 p;
    int32_t row[J];
    bool there[J];
    int lane, col, quad, eighth, piece;

    __device__ __forceinline__ Tile()
        : lane(threadIdx.x % kWave), col(lane % 16), quad(lane / 16), eighth(lane / 8),
          piece(lane % 8)
    {
    }
    // rows from the tile's `skip`-th on; false: there are none
    __device__ __forceinline__ bool take(const PassArgs &a, int64_t tile, int skip = 0)
    {
        if (a.tiles) {
            p = a.tiles[tile];
            p.first += skip;
            p.count -= skip;
            if (p.group < 0 || p.count <= 0)
                return false;
        } else {
            const int32_t id = a.ids[tile];
            p = {id >= 0 && id < a.groups ? id : a.groups, (int32_t)tile, 1, 0};
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int32_t at = j * 8 + eighth;
            there[j] = at < p.count;                      // (others read the tile's first row)
            const int32_t place = p.first + (there[j] ? at : 0);
            row[j] = a.order ? a.order[place] : place;
        }
        return true;
    }
    // rows from the tile's `skip`-th on or, where there are none (false), its first
    __device__ __forceinline__ bool take_or_first(const PassArgs &a, int64_t tile, int skip)
    {
        const bool any = take(a, tile, a.tiles ? skip : 0) && (a.tiles || skip == 0);
        if (!any && p.group >= 0) {
            if (a.tiles)
                take(a, tile);
#pragma unroll
            for (int j = 0; j < J; ++j)
                there[j] = false;
        }
        return any;
    }
    // as take(), of 16 rows: a lane's is l % 16.  Rows may be fewer than none: of tiles alone
    // is said that there are none
    __device__ __forceinline__ bool take_lanes(const PassArgs &a, int64_t tile, int skip)
    {
        p = a.tiles[tile];
        if (p.group < 0)
            return false;
        p.first += skip;
        p.count -= skip;
        there[0] = col < p.count;
        row[0] = there[0] ? a.order[p.first + col] : 0;
        return true;
    }
    // of row 16 rt + l % 16
    __device__ __forceinline__ int32_t sample(int rt) const
    {
        const int from = col % 8 * 8;
        const int32_t low = __shfl(row[2 * rt], from), high = __shfl(row[2 * rt + 1], from);
        return col < 8 ? low : high;
    }
    __device__ __forceinline__ bool sample_there(int rt) const { return rt * 16 + col < p.count; }
};

// E terms, `step` elements apart, of a matrix in LDS.
template <int W>
__device__ __forceinline__ Frag lds_across(const char *p, int at, int step)
{
    Frag f;
    if constexpr (kSize<W> == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            f.w[e] = reinterpret_cast<const uint32_t *>(p)[at + e * step];
    } else {
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = reinterpret_cast<const uint16_t *>(p)[at + e * step];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f.w[i] = v[2 * i] | v[2 * i + 1] << 16;
    }
    return f;
}

// h += w1 x over terms [from, to): units of 128 bytes of a row; `to` is k or a multiple of the
// unit.  A unit's loads are issued before the products of the one before.  A wave's units are
// neighbours: rows need not start at a cache line, and a line that two waves ask for at a time
// stalls the L1 until it is there.
template <int W, int X, int CT, int RT, bool BACK>
__device__ __forceinline__ void shrink(const PassArgs &a, const Tile<RT> &tile, char *lds,
                                       int32_t from, int32_t to, f32x4 (&h)[RT][CT])
{
    constexpr int E = kEls<W>, S = kSize<W>, kUnit = 8 * E, J = 2 * RT, C = 2 * CT;
    char *lds_w = lds + RT * 16 * 128;
    const char *x[J], *w[BACK ? 1 : C];
#pragma unroll
    for (int j = 0; j < J; ++j)
        x[j] = a.x + tile.row[j] * a.x_stride + tile.piece * 16;
    const char *first = a.w1 + tile.p.group * a.w1_step;
    if constexpr (!BACK) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            // ranks behind the last one read its weights: what comes of it is cleared afterwards
            const int32_t r = min(c * 8 + tile.eighth, a.rank - 1);
            w[c] = first + (int64_t)r * a.k * S + tile.piece * 16;
        }
    }
    const int32_t pieces = 8 * a.rank;                    // BACK: of a unit's weights
    const int64_t across = (int64_t)a.rank * S;
    struct Unit {
        Frag x[J], w[C];
    };
    const auto load = [&](Unit &u, int32_t k0) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < J; ++j)
            u.x[j] = load_16(x[j] + (int64_t)k0 * S);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (!BACK) {
                u.w[c] = load_16(w[c] + (int64_t)k0 * S);
            } else {
                const int at = c * kWave + tile.lane;
                if (at < pieces)
                    u.w[c] = load_16(first + k0 * across + at * 16);
            }
        }
    };
    const auto put = [&](const Unit &u) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < J; ++j)
            lds_put(lds + slot_at(j * 8 + tile.eighth, tile.piece), to_terms<X>(u.x[j]));
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (!BACK) {
                lds_put(lds_w + slot_at(c * 8 + tile.eighth, tile.piece), u.w[c]);
            } else {
                const int at = c * kWave + tile.lane;
                if (at < pieces)
                    lds_put(lds_w + at * 16, u.w[c]);
            }
        }
    };
    const auto products = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            Frag fx[RT], fw[CT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                fx[rt] = lds_frag(lds + slot_at(rt * 16 + tile.col, half * 4 + tile.quad));
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                if constexpr (!BACK) {
                    fw[ct] = lds_frag(lds_w + slot_at(ct * 16 + tile.col, half * 4 + tile.quad));
                } else {
                    const int32_t r = min(ct * 16 + tile.col, a.rank - 1);
                    fw[ct] = lds_across<W>(lds_w, (half * 4 + tile.quad) * E * a.rank + r, a.rank);
                }
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
                    h[rt][ct] = mma<W>(fw[ct], fx[rt], h[rt][ct]);
        }
    };
    const int32_t whole = min(to, a.k / kUnit * kUnit);
    int32_t k0 = from;
    if (k0 < whole) {
        Unit u;
        load(u, k0);
        for (;;) {
            put(u);
            rows::wave_sync();
            k0 += kUnit;
            const bool more = k0 < whole;
            if (more)
                load(u, k0);
            products();
            rows::wave_sync();
            if (!more)
                break;
        }
    }
    if (k0 < to) {                                        // the row's last terms, zeros after them
        const int32_t left = a.k - k0 - tile.piece * E;
#pragma unroll
        for (int j = 0; j < J; ++j)
            lds_put(lds + slot_at(j * 8 + tile.eighth, tile.piece),
                    to_terms<X>(load_frag<W>(x[j] + (int64_t)k0 * S, left, a.k)));
        if constexpr (!BACK) {
#pragma unroll 1
            for (int c = 0; c < C; ++c) {
                const int32_t r = min(c * 8 + tile.eighth, a.rank - 1);
                lds_put(lds_w + slot_at(c * 8 + tile.eighth, tile.piece),
                        load_frag<W>(first + ((int64_t)r * a.k + k0) * S + tile.piece * 16, left,
                                     a.k));
            }
        } else {
            const int32_t there = (a.k - k0) * a.rank;
#pragma unroll 1
            for (int at = tile.lane; at < pieces; at += kWave)
                lds_put(lds_w + at * 16, load_frag<W>(first + k0 * across + at * 16,
                                                      there - at * E, (int64_t)a.k * a.rank));
        }
        rows::wave_sync();
        products();
        rows::wave_sync();
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

// Ranks r .. r + 3 of a row of h, as many as there are.
__device__ __forceinline__ void store_ranks(float *row, int32_t r, int32_t rank, f32x4 v)
{
    if (r + 4 <= rank) {
        __builtin_memcpy(row + r, &v, 16);
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (r + i < rank)
            row[r + i] = v[i];
}
__device__ __forceinline__ f32x4 load_ranks(const float *row, int32_t r, int32_t rank)
{
    f32x4 v = {0, 0, 0, 0};
    if (r + 4 <= rank) {
        __builtin_memcpy(&v, row + r, 16);
        return v;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (r + i < rank)
            v[i] = row[r + i];
    return v;
}

template <int RT, int CT>
__device__ __forceinline__ void store_hidden(float *to, int32_t rank, const Tile<RT> &tile,
                                             const f32x4 (&h)[RT][CT])
{
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int32_t row = tile.sample(rt);
        if (tile.sample_there(rt))
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
                store_ranks(to + (int64_t)row * rank, ct * 16 + tile.quad * 4, rank, h[rt][ct]);
    }
}

// ---- the second product, by 16 rows a wave ----
// Its weights in LDS.  Forward: a column's ranks, a multiple of four (zeros past the last), in an
// odd number of 16-byte slots, so that 16 columns are in different banks; back: a rank's columns.
template <int W, int CT, bool BACK>
struct Second {
    static constexpr int E = kEls<W>, S = kSize<W>;
    static constexpr int kCols = BACK ? 16 * E : 8 * E;   // a unit: columns whose sums a wave holds
    static constexpr int T = kCols / 16;
    static constexpr int kPitch = kCols + 4;              // floats of a row of a unit's sums
    const char *lds;
    int pitch, rank, col, quad;                           // pitch: bytes

    // 4 ranks of column m + t 16 + l % 16 (forward) or m + t + E (l % 16) (back), zeros past the
    // last rank
    __device__ __forceinline__ void terms_of(int m, int ct, uint32_t (&v)[T][S], int there) const
    {
        const int r = ct * 16 + quad * 4;
        if constexpr (!BACK) {
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const char *at = lds + (m + t * 16 + col) * pitch + r * S;
#pragma unroll
                for (int i = 0; i < S; ++i)
                    v[t][i] = 0;
                if (r < rank && t * 16 < there)
                    __builtin_memcpy(v[t], __builtin_assume_aligned(at, 4 * S), 4 * S);
            }
        } else {
            Frag f[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[i] = lds_frag(lds + min(r + i, rank - 1) * pitch + (m + col * E) * S);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    f[i].w[e] = r + i < rank ? f[i].w[e] : 0;
            }
#pragma unroll
            for (int t = 0; t < T; ++t) {
                if constexpr (S == 4) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[t][i] = f[i].w[t];
                } else {
                    const uint32_t pick = t & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        v[t][i] = __builtin_amdgcn_perm(f[2 * i + 1].w[t / 2],
                                                        f[2 * i].w[t / 2], pick);
                }
            }
        }
    }
    // factor w2 h of columns [m, m + kCols) to sums [16 rows][pitch floats], from column 0 on;
    // forward, as many 16s of them as the first `there` are in.
    __device__ __forceinline__ void unit(int m, const Frag (&terms)[CT], float factor, float *sums,
                                         int sums_pitch, int there = kCols) const
    {
        f32x4 sum[T];
#pragma unroll
        for (int t = 0; t < T; ++t)
            sum[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            uint32_t v[T][S];
            terms_of(m, ct, v, there);
#pragma unroll
            for (int t = 0; t < T; ++t)
                sum[t] = mma_h<W>(v[t], terms[ct], sum[t]);
        }
        float *own = sums + col * sums_pitch;             // the lane's row
        if constexpr (!BACK) {
#pragma unroll
            for (int t = 0; t < T; ++t)
                if (t * 16 < there)
                    *reinterpret_cast<f32x4 *>(own + t * 16 + quad * 4) = sum[t] * factor;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int q = 0; q < E / 4; ++q) {
                    f32x4 v;
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        v[u] = sum[q * 4 + u][i] * factor;
                    *reinterpret_cast<f32x4 *>(own + (quad * 4 + i) * E + q * 4) = v;
                }
        }
    }
};

__device__ __forceinline__ int odd_slots(int bytes) { return (((bytes + 15) / 16) | 1) * 16; }

// v += base_scale * base, E columns of it; b: its bits.
template <int W>
__device__ __forceinline__ void add_base(const PassArgs &a, float (&v)[kEls<W>], const Frag &b)
{
#pragma unroll
    for (int u = 0; u < kEls<W>; ++u) {
        float c;
        if constexpr (W == kF32)
            c = a.base_i32 ? (float)(int32_t)b.w[u] : __uint_as_float(b.w[u]);
        else if constexpr (W == kBf16)
            c = __uint_as_float(u & 1 ? b.w[u / 2] & 0xFFFF0000u : b.w[u / 2] << 16);
        else
            c = (float)__builtin_bit_cast(_Float16, (uint16_t)(b.w[u / 2] >> (16 * (u & 1))));
        v[u] += a.base_scale * c;
    }
}

// E results to memory, or as many as there are.
template <int W>
__device__ __forceinline__ void store_row(char *to, const float (&v)[kEls<W>], int32_t left)
{
    constexpr int E = kEls<W>, S = kSize<W>;
    if (left >= E) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = S == 4 ? el_bits<W>(v[i])
                          : el_bits<W>(v[2 * i % E]) | el_bits<W>(v[(2 * i + 1) % E]) << 16;
        __builtin_memcpy(to, w, 16);
        return;
    }
#pragma unroll
    for (int u = 0; u < E; ++u)
        if (u < left) {
            if constexpr (S == 4)
                reinterpret_cast<uint32_t *>(to)[u] = el_bits<W>(v[u]);
            else
                reinterpret_cast<uint16_t *>(to)[u] = (uint16_t)el_bits<W>(v[u]);
        }
}

// Four ranks of a column of up [m][rank], zeros past the last.
template <int W>
__device__ __forceinline__ void load_four(const char *p, int left, uint32_t (&v)[kSize<W>])
{
    constexpr int S = kSize<W>;
    if (left >= 4) {
        __builtin_memcpy(v, p, 4 * S);
        return;
    }
#pragma unroll
    for (int i = 0; i < S; ++i)
        v[i] = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < left) {
            if constexpr (S == 4)
                v[i] = reinterpret_cast<const uint32_t *>(p)[i];
            else
                v[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << (16 * (i & 1));
        }
}

// ---- narrow adapters: 16 rows a wave, whole rows at a time ----
// (2^18 rows of 100 int32 counts and logits in the order of 24 adapters, rank 8: 93 us for 316 MB;
// a block's loads, products and stores take turns, and LDS and registers leave room for four.
// Loads that pass by the L1: 85 us, 109 without, inputs warm.)
// A block has a tile, and its adapter in LDS.  A wave copies its 16 rows of x there, and holds
// those of base in registers meanwhile, by 16-byte pieces in the order of memory: of the lines at
// the ends of rows, none is asked for twice.
constexpr int kTileWaves = kTile / 16;

// e / d for e < 2^13, d <= 2^7.
struct Divide {
    uint32_t magic;
    __device__ __forceinline__ explicit Divide(int d) : magic(((1u << 20) + d - 1) / d) {}
    __device__ __forceinline__ int operator()(int e) const { return (int)(e * magic >> 20); }
};

// `rows` rows of n elements, `stride` bytes apart, to LDS rows of `pitch` bytes, zeros to the end
// of their last pieces; by all of a block.
template <int W>
__device__ __forceinline__ void stage_rows(char *to, int pitch, const char *from, int64_t stride,
                                           int rows, int n)
{
    constexpr int E = kEls<W>;
    const int pieces = n / E;
    if (pieces > 0) {
        const Divide row_of(pieces);
#pragma unroll 4
        for (int at = threadIdx.x; at < rows * pieces; at += kTileWaves * kWave) {
            const int r = row_of(at), p = at - r * pieces;
            lds_put(to + r * pitch + p * 16, load_16(from + r * stride + p * 16));
        }
    }
    if (n % E)
#pragma unroll 1
        for (int r = threadIdx.x; r < rows; r += kTileWaves * kWave)
            lds_put(to + r * pitch + pieces * 16,
                    load_frag<W>(from + r * stride + pieces * 16, n % E, n));
}

// up [m][rank] of `cols` columns to LDS, a column in `pitch` bytes; by all of a block.
template <int W>
__device__ __forceinline__ void stage_up(char *to, int pitch, const char *from, int rank, int cols)
{
    constexpr int S = kSize<W>;
    if (rank * S % 16 == 0) {
        stage_rows<W>(to, pitch, from, (int64_t)rank * S, cols, rank);
        return;
    }
    const int fours = (rank + 3) / 4;
    const Divide col_of(fours);
#pragma unroll 2
    for (int at = threadIdx.x; at < cols * fours; at += kTileWaves * kWave) {
        const int m = col_of(at), r = (at - m * fours) * 4;
        uint32_t v[S];
        load_four<W>(from + (m * rank + r) * S, rank - r, v);
        __builtin_memcpy(__builtin_assume_aligned(to + m * pitch + r * S, 4 * S), v, 4 * S);
    }
}

// LDS of a block: the first product's weights, the second's, and a wave's rows of x, later its
// sums.
template <int W, bool BACK>
struct NarrowRoom {
    int w1_pitch, w2_pitch, x_pitch, sums_pitch;          // bytes; sums_pitch floats
    int w1, w2, wave;                                     // bytes

    __host__ __device__ NarrowRoom(int k, int m, int rank)
    {
        // (in whole units, 100 floats take 43 KB and 3 blocks a CU fit)
        constexpr int E = kEls<W>, S = kSize<W>, kCols = BACK ? 16 * E : 16;
        const auto odd = [](int bytes) { return (((bytes + 15) / 16) | 1) * 16; };
        const int cols = (m + kCols - 1) / kCols * kCols;
        x_pitch = odd(k * S);
        sums_pitch = cols + 4;
        w1_pitch = odd(k * S);
        w2_pitch = BACK ? odd(cols * S) : odd(rank * S);
        w1 = BACK ? ((k + E - 1) / E * E * rank * S + 15) / 16 * 16 : rank * w1_pitch;
        w2 = BACK ? rank * w2_pitch : cols * w2_pitch;
        const int sums = 16 * sums_pitch * 4, x = 16 * x_pitch;
        wave = sums > x ? sums : x;
    }
    __host__ __device__ int bytes() const { return w1 + w2 + kTileWaves * wave; }
};

template <int W, int X, int CT, bool BACK>
__global__ __launch_bounds__(kTileWaves * kWave, CT <= 2 ? 4 : 2) void k_narrow(PassArgs a)
{
    constexpr int E = kEls<W>, S = kSize<W>, F = 8;       // pieces of 16 rows: 512 at most
    extern __shared__ __align__(16) char lds[];
    const NarrowRoom<W, BACK> room(a.k, a.m, a.rank);
    char *w1 = lds, *w2 = lds + room.w1;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    char *own = lds + room.w1 + room.w2 + wave * room.wave;
    Tile<1> tile;
    if (!tile.take_lanes(a, blockIdx.x, wave * 16))
        return;                                           // (the whole block)
    const bool adapted = tile.p.group < a.groups;
    const int x_pieces = a.k / E, m_pieces = a.m / E;
    const Divide x_row(max(x_pieces, 1)), m_row(max(m_pieces, 1));
    Frag b[F], b_end = {{0, 0, 0, 0}};
    const bool end_lane = tile.lane < tile.p.count && tile.lane < 16;
    if (!BACK && a.base && a.out) {
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const int at = i * kWave + tile.lane, r = m_row(at), p = at - r * m_pieces;
            const int32_t row = __shfl(tile.row[0], r);
            if (r < tile.p.count && at < 16 * m_pieces)
                b[i] = load_nt(a.base + row * a.base_stride + p * 16);
        }
        if (end_lane && a.m % E)
            b_end = load_frag<W>(a.base + tile.row[0] * a.base_stride + m_pieces * 16, a.m % E,
                                 a.m);
    }
    f32x4 h[1][CT];
    clear(h);
    if (adapted) {
        const char *down = a.w1 + tile.p.group * a.w1_step, *up = a.w2 + tile.p.group * a.w2_step;
        Frag x[F];
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const int at = i * kWave + tile.lane, r = x_row(at), p = at - r * x_pieces;
            const int32_t row = __shfl(tile.row[0], r);
            if (r < tile.p.count && at < 16 * x_pieces)
                x[i] = load_nt(a.x + row * a.x_stride + p * 16);
        }
        if constexpr (!BACK) {
            stage_rows<W>(w1, room.w1_pitch, down, (int64_t)a.k * S, a.rank, a.k);
            if (a.out)
                stage_up<W>(w2, room.w2_pitch, up, a.rank, a.m);
        } else {
            const int there = a.k * a.rank;               // [k][rank] as it lies, zeros behind
#pragma unroll 2
            for (int at = threadIdx.x; at * 16 < room.w1; at += kTileWaves * kWave)
                lds_put(w1 + at * 16, load_frag<W>(down + at * 16, there - at * E, there));
            if (a.out)
                stage_rows<W>(w2, room.w2_pitch, up, (int64_t)a.m * S, a.rank, a.m);
        }
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const int at = i * kWave + tile.lane, r = x_row(at), p = at - r * x_pieces;
            if (r < tile.p.count && at < 16 * x_pieces)
                lds_put(own + r * room.x_pitch + p * 16, to_terms<X>(x[i]));
        }
        if (end_lane && a.k % E)
            lds_put(own + tile.lane * room.x_pitch + x_pieces * 16,
                    to_terms<X>(load_frag<W>(a.x + tile.row[0] * a.x_stride + x_pieces * 16,
                                             a.k % E, a.k)));
        __syncthreads();
        // (rows that are not there: whatever is in LDS, in columns of their own)
        const int pieces = (a.k + E - 1) / E;
        for (int p0 = 0; p0 < pieces; p0 += 4) {
            const int p = p0 + tile.quad;
            Frag fx = {{0, 0, 0, 0}}, fw[CT];
            if (p < pieces)
                fx = lds_frag(own + tile.col * room.x_pitch + p * 16);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const int r = min(ct * 16 + tile.col, a.rank - 1);
                fw[ct] = {{0, 0, 0, 0}};
                if (p < pieces) {
                    if constexpr (!BACK)
                        fw[ct] = lds_frag(w1 + r * room.w1_pitch + p * 16);
                    else
                        fw[ct] = lds_across<W>(w1, p * E * a.rank + r, a.rank);
                }
                h[0][ct] = mma<W>(fw[ct], fx, h[0][ct]);
            }
        }
        clear_past_rank(a.rank, tile.quad, h);
        rows::wave_sync();
    }
    if (a.hidden && tile.col < tile.p.count)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
            store_ranks(a.hidden + (int64_t)tile.row[0] * a.rank, ct * 16 + tile.quad * 4, a.rank,
                        h[0][ct]);
    if (!a.out)
        return;
    float *sums = reinterpret_cast<float *>(own);
    if (adapted) {
        typedef Second<W, CT, BACK> Product;
        const Product second = {w2, room.w2_pitch, a.rank, tile.col, tile.quad};
        Frag terms[1][CT];
        float factor[1];
        make_terms<W>(h, terms, factor);
        factor[0] *= a.scales ? a.scales[tile.p.group] : a.scale;
#pragma unroll 1
        for (int m = 0; m < a.m; m += Product::kCols)
            second.unit(m, terms[0], factor[0], sums + m, room.sums_pitch, a.m - m);
        rows::wave_sync();
    }
    const auto result = [&](int r, int p, const Frag &base, float (&v)[E]) __attribute__((always_inline)) {
        if (adapted) {
            __builtin_memcpy(v, sums + r * room.sums_pitch + p * E, sizeof v);
        } else {
#pragma unroll
            for (int u = 0; u < E; ++u)
                v[u] = 0.0f;
        }
        if (!BACK && a.base)
            add_base<W>(a, v, base);
    };
#pragma unroll
    for (int i = 0; i < F; ++i) {
        const int at = i * kWave + tile.lane, r = m_row(at), p = at - r * m_pieces;
        const int32_t row = __shfl(tile.row[0], r);
        if (r < tile.p.count && at < 16 * m_pieces) {
            float v[E];
            result(r, p, b[i], v);
            store_row<W>(a.out + row * a.out_stride + p * 16, v, E);
        }
    }
    if (end_lane && a.m % E) {
        float v[E];
        result(tile.lane, m_pieces, b_end, v);
        store_row<W>(a.out + tile.row[0] * a.out_stride + m_pieces * 16, v, a.m % E);
    }
}

// ---- wide adapters ----
// waves that share a block's terms: as many as a rank's weights leave LDS for
template <int CT> constexpr int kTermWaves = CT <= 2 ? 8 : 4;
// waves a SIMD to compile for; k_expand's: what its LDS leaves room for
template <int CT> constexpr int kWavesPerSimd = CT <= 2 ? 4 : CT == 4 ? 3 : 2;
template <int W, int CT, bool BACK>
constexpr int kExpandWaves = !BACK || (kSize<W> == 4 && CT < 8) ? kWavesPerSimd<CT>
                             : CT <= 2 ? 3 : CT == 4 ? 2 : 1;

// Part `blockIdx % splits` of the h of 32 rows of a tile, to [part][row][rank].
//
// Bound by the memory's answers to 128-byte pieces of many rows: 20 us for 50 MB (12289 x 2048
// bfloat16, rank 24), 47 us for 123 MB of odd rows (back; the loads alone take 26).  64 rows a wave,
// loads two units ahead and other numbers of blocks were within 3% or slower.
template <int W, int X, int CT, int RT, bool BACK>
__global__ __launch_bounds__(kTermWaves<CT> * kWave, kWavesPerSimd<CT>) void k_shrink(PassArgs a)
{
    constexpr int NW = kTermWaves<CT>, kAcc = CT * RT * 4, kUnit = 8 * kEls<W>;
    constexpr int kWaveBytes = (RT + CT) * 16 * 128;
    static_assert(kAcc * kWave * 4 <= kWaveBytes, "sums fit where the terms were");
    __shared__ __align__(16) char lds[NW * kWaveBytes];
    float *joined = reinterpret_cast<float *>(lds);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int64_t at = blockIdx.x / a.splits;
    const int part = (int)(blockIdx.x - at * a.splits);
    constexpr int kParts = RT == 2 ? kTile / 32 : 1;
    Tile<RT> tile;
    if (!tile.take(a, at / kParts, (int)(at % kParts) * 32))
        return;
    const bool adapted = tile.p.group < a.groups;
    if (adapted) {
        f32x4 h[RT][CT];
        clear(h);
        const int32_t units = (a.k + kUnit - 1) / kUnit, shares = a.splits * NW;
        const int32_t each = (units + shares - 1) / shares, share = part * NW + wave;
        const int32_t from = min(share * each, units) * kUnit;
        const int32_t to = min(min((share + 1) * each, units) * kUnit, a.k);
        shrink<W, X, CT, RT, BACK>(a, tile, lds + wave * kWaveBytes, from, to, h);
        clear_past_rank(a.rank, tile.quad, h);
        // the waves' sums, added in order; each wave adds up some of them
        __syncthreads();
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    joined[(wave * kAcc + (rt * CT + ct) * 4 + i) * kWave + tile.lane] =
                        h[rt][ct][i];
        __syncthreads();
    }
    // wave w stores fragments w, w + NW, ... of the tile's RT * CT
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int32_t row = tile.sample(rt);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int f = rt * CT + ct;
            if (f % NW != wave)
                continue;
            f32x4 sum = {0, 0, 0, 0};
            if (adapted)
#pragma unroll
                for (int w = 0; w < NW; ++w)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sum[i] += joined[(w * kAcc + f * 4 + i) * kWave + tile.lane];
            if (tile.sample_there(rt))
                store_ranks(a.partial + ((int64_t)part * a.n_rows + row) * a.rank,
                            ct * 16 + tile.quad * 4, a.rank, sum);
        }
    }
}

// Units of columns of a tile, 16 rows a wave; a unit's weights are in LDS for all of them, the
// next unit's on their way.
//
// Bound by memory in this pattern: 71 us for 246 MB (12289 x 5003 bfloat16, rank 24) and 46 us for
// 134 MB (8192 x 4096 float16, rank 64), where loads and stores alone take 75 and 35 us (by units)
// and a copy of whole rows 48 and 26.
// Units at a time: two where their registers leave four waves a SIMD (12289 rows, 5003 columns,
// rank 24: 71 us, by one 87; rank 64, 8192 rows of 4096: 58 us, by one 49).
template <int CT, bool BACK> constexpr int kUnits = BACK || CT > 2 ? 1 : 2;

template <int W, int CT, bool BACK>
__global__ __launch_bounds__(kTileWaves * kWave, (kExpandWaves<W, CT, BACK>))
void k_expand(PassArgs a, int32_t blocks)
{
    typedef Second<W, CT, BACK> Product;
    constexpr int E = kEls<W>, S = kSize<W>, kUnit = Product::kCols, J = 2, U = kUnits<CT, BACK>;
    constexpr int kCols = U * kUnit;
    constexpr int kWeights = BACK ? CT * 16 * (kCols * S + 16)
                                  : kCols * ((CT * 16 * S / 16) | 1) * 16;
    constexpr int kPieces = (CT * 16 * kCols * S / 16 + 255) / 256;   // of the weights, a lane
    __shared__ __align__(16) char weights[2][kWeights];
    __shared__ __align__(16) float sums[kTileWaves][16 * Product::kPitch];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int64_t at = blockIdx.x / blocks;
    const int block = (int)(blockIdx.x - at * blocks);
    Tile<1> tile;
    // (a wave without rows takes the tile's first one, and stores nothing)
    const bool any = tile.take_or_first(a, at, wave * 16);
    if (tile.p.group < 0)
        return;
    const bool adapted = tile.p.group < a.groups;
    const int32_t units = (a.m + kUnit - 1) / kUnit, each = (units + blocks - 1) / blocks * kUnit;
    const int32_t from = block * each, to = a.out ? min(from + each, a.m) : 0;
    Frag b[U][J], b_next[U][J];
    const auto load_base = [&](Frag (&f)[U][J], int32_t m0) __attribute__((always_inline)) {
        if constexpr (!BACK) {
            if (!a.base || !any)
                return;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int32_t m = m0 + u * kUnit + tile.piece * E;
                const char *at = a.base + (int64_t)m * S;
                if (m0 + (u + 1) * kUnit <= a.m) {
#pragma unroll
                    for (int j = 0; j < J; ++j)
                        f[u][j] = load_16(at + tile.row[j] * a.base_stride);
                } else if (m0 + u * kUnit < to) {
#pragma unroll
                    for (int j = 0; j < J; ++j)
                        f[u][j] = load_frag<W>(at + tile.row[j] * a.base_stride, a.m - m, a.m);
                }
            }
        }
    };
    if (from < to)
        load_base(b, from);
    // the weights of a unit: pieces to registers, and from there to LDS
    const char *w2 = a.w2 + (adapted ? tile.p.group * a.w2_step : 0);
    const int pitch = BACK ? kCols * S + 16 : odd_slots(a.rank * S);
    const bool by_pieces = BACK || a.rank * S % 16 == 0;
    const int per = BACK ? kCols * S / 16 : max(a.rank * S / 16, 1);  // pieces of an LDS row
    const Divide row_of(per);
    Frag w[kPieces];
    const auto load_weights = [&](int32_t m0) __attribute__((always_inline)) {
        if (!adapted || !by_pieces)
            return;
        const int all = BACK ? a.rank * per : min(to - m0, kCols) * per;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int e = i * kTileWaves * kWave + threadIdx.x, r = row_of(e), p = e - r * per;
            if (e < all) {
                if constexpr (BACK)
                    w[i] = load_frag<W>(w2 + ((int64_t)r * a.m + m0) * S + p * 16,
                                        a.m - m0 - p * E, a.m);
                else
                    w[i] = load_16(w2 + (int64_t)m0 * a.rank * S + e * 16);
            }
        }
    };
    const auto put_weights = [&](int32_t m0, char *to_lds) __attribute__((always_inline)) {
        if (!adapted)
            return;
        if (!BACK && !by_pieces) {
            stage_up<W>(to_lds, pitch, w2 + (int64_t)m0 * a.rank * S, a.rank, min(to - m0, kCols));
            return;
        }
        const int all = BACK ? a.rank * per : min(to - m0, kCols) * per;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int e = i * kTileWaves * kWave + threadIdx.x, r = row_of(e), p = e - r * per;
            if (e < all)
                lds_put(to_lds + r * pitch + p * 16, w[i]);
        }
    };
    if (from < to)
        load_weights(from);
    f32x4 h[1][CT];
    clear(h);
    const int64_t row = tile.sample(0);
#pragma unroll CT <= 2 ? 4 : 2
    for (int32_t p = 0; p < a.splits; ++p)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
            h[0][ct] += load_ranks(a.partial + (p * a.n_rows + row) * a.rank,
                                   ct * 16 + tile.quad * 4, a.rank);
    if (a.hidden && a.hidden != a.partial && block == 0 && any)
        store_hidden(a.hidden, a.rank, tile, h);
    if (from >= to)
        return;
    Frag terms[1][CT];
    float factor[1];
    make_terms<W>(h, terms, factor);
    factor[0] *= !adapted ? 0.0f : a.scales ? a.scales[tile.p.group] : a.scale;
    put_weights(from, weights[0]);
    int turn = 0;
    for (int32_t m0 = from; m0 < to; m0 += kCols, turn ^= 1) {
        // this unit's weights are there, and nobody reads those of the one before
        __syncthreads();
        const int32_t next = m0 + kCols;
        if (next < to) {
            load_weights(next);
            load_base(b_next, next);
        }
        if (any) {
            float *own = sums[wave];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int32_t mu = m0 + u * kUnit;
                if (mu >= to)
                    break;
                if (adapted) {
                    const Product second = {weights[turn], pitch, a.rank, tile.col, tile.quad};
                    second.unit(u * kUnit, terms[0], factor[0], own, Product::kPitch);
                }
                rows::wave_sync();
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int q = 0; q < (BACK ? 2 : 1); ++q) {
                        const int c = (tile.piece + q * 8) * E;
                        float v[E];
                        if (adapted) {
                            __builtin_memcpy(v, own + (j * 8 + tile.eighth) * Product::kPitch + c,
                                             sizeof v);
                        } else {
#pragma unroll
                            for (int i = 0; i < E; ++i)
                                v[i] = 0.0f;
                        }
                        if (!BACK && a.base)
                            add_base<W>(a, v, b[u][j]);
                        if (tile.there[j])
                            store_row<W>(a.out + tile.row[j] * a.out_stride +
                                         (int64_t)(mu + c) * S, v, a.m - mu - c);
                    }
                rows::wave_sync();
            }
        }
        if (next < to) {
            put_weights(next, weights[turn ^ 1]);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < J; ++j)
                    b[u][j] = b_next[u][j];
        }
    }
}

template <int W, int X, int CT, bool BACK>
hipError_t pass_of(const PassArgs &a, hipStream_t stream)
{
    if (a.splits == 0) {
        const NarrowRoom<W, BACK> room(a.k, a.m, a.rank);
        hipLaunchKernelGGL((k_narrow<W, X, CT, BACK>), dim3((uint32_t)a.n_tiles),
                           dim3(kTileWaves * kWave), room.bytes(), stream, a);
        return hipGetLastError();
    }
    const dim3 term_waves(kTermWaves<CT> * kWave);
    if (a.tiles)
        hipLaunchKernelGGL((k_shrink<W, X, CT, 2, BACK>),
                           dim3((uint32_t)(a.n_tiles * (kTile / 32) * a.splits)), term_waves, 0,
                           stream, a);
    else
        hipLaunchKernelGGL((k_shrink<W, X, CT, 1, BACK>), dim3((uint32_t)(a.n_tiles * a.splits)),
                           term_waves, 0, stream, a);
    if (hipError_t err = hipGetLastError(); err != hipSuccess)
        return err;
    if (!a.out && a.hidden == a.partial)
        return hipSuccess;
    static_assert(Second<W, CT, BACK>::kCols * kSize<W> == (BACK ? 256 : 128), "expand_blocks()");
    const int32_t blocks = expand_blocks(a, kSize<W>, BACK);
    hipLaunchKernelGGL((k_expand<W, CT, BACK>), dim3((uint32_t)(a.n_tiles * blocks)),
                       dim3(kTileWaves * kWave), 0, stream, a, blocks);
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
//
// Bound by the waves' chains of loads: 50 us for 173 MB (12289 rows of 2048 and 5003 bfloat16 columns,
// rank 24), 58 without the next step's row numbers ahead and with odd rows' ends element by
// element; h through LDS instead 69.
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
    const int32_t c0 = block * 16 * E, at = c0 + col * E, left = j.cols - at;
    const bool whole_block = c0 + 16 * E <= j.cols;
    f32x4 sum[CT][E];
    clear(sum);
    const char *y = j.y + (int64_t)at * S;
    const int32_t *order = a.order + p.first;
    const auto rows_of = [&](int32_t s, int32_t (&row)[kRows]) __attribute__((always_inline)) {
        if (s + kStep <= p.count) {
            __builtin_memcpy(row, order + s + quad * kRows, sizeof row);
        } else {
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                row[u] = order[min(s + quad * kRows + u, p.count - 1)];
        }
    };
    int32_t next[kRows];
    rows_of(wave * kStep, next);
    for (int32_t s = wave * kStep; s < p.count; s += NW * kStep) {
        const bool whole_step = s + kStep <= p.count;
        Frag f[kRows];
        float hv[CT][kRows];
        int32_t row[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u)
            row[u] = next[u];
        if (whole_block) {
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                __builtin_memcpy(f[u].w, y + row[u] * j.y_stride, 16);
        } else {
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                f[u] = load_frag<W>(y + row[u] * j.y_stride, left, j.cols);
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int32_t r = min(ct * 16 + col, a.rank - 1);   // (past the rank: not stored)
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                hv[ct][u] = j.h[(int64_t)row[u] * a.rank + r];
        }
        rows_of(s + NW * kStep, next);                    // the next step's, meanwhile
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
            if (left >= E) {
                __builtin_memcpy(to, v, sizeof v);
                continue;
            }
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
// added in order; those of down and of up by blocks of their own.
template <int W>
__global__ __launch_bounds__(256) void k_join_grads(GradArgs a, int32_t per_group)
{
    const int32_t k = (int32_t)(blockIdx.x / ((uint32_t)a.groups * per_group));
    const int32_t block = (int32_t)(blockIdx.x - (uint32_t)k * a.groups * per_group);
    const int32_t g = block / per_group;
    const GradJob &j = a.job[k];
    if (!j.out || (a.chunk_starts && a.chunk_starts[g + 1] - a.chunk_starts[g] == 1))
        return;
    const int32_t first = a.chunk_starts ? a.slot_starts[g] : 0,
                  last = a.chunk_starts ? a.slot_starts[g + 1] : 0;
    const float scale = a.scales ? a.scales[g] : a.scale;
    const int64_t all = (int64_t)a.rank * j.cols;
    for (int64_t e = (int64_t)(block - g * per_group) * 256 + threadIdx.x; e < all;
         e += (int64_t)per_group * 256) {
        float v = 0.0f;
#pragma unroll 8
        for (int32_t c = first; c < last; ++c)
            v += j.partial[c * all + e];
        int64_t to = g * all + e;
        if (j.transposed) {
            const int64_t r = e / j.cols, at = e - r * j.cols;
            to = g * all + at * a.rank + r;
        }
        if constexpr (kSize<W> == 4)
            reinterpret_cast<uint32_t *>(j.out)[to] = el_bits<W>(scale * v);
        else
            reinterpret_cast<uint16_t *>(j.out)[to] = (uint16_t)el_bits<W>(scale * v);
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
    hipLaunchKernelGGL(k_join_grads<W>, dim3((uint32_t)(2 * (int64_t)a.groups * per_group)),
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
bool fits_narrow(int32_t k, int32_t m, int32_t rank, bool back)
{
    const int64_t row = (int64_t)std::max(k, m) * kSize<W>;
    return row <= 512 && (back ? NarrowRoom<W, true>(k, m, rank).bytes()
                               : NarrowRoom<W, false>(k, m, rank).bytes()) <= 64 << 10;
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
