// Kernels of low-rank adapters (internal), included once for each weight type W (float32,
// float16, bfloat16); x of type X, W or int32.
//
// A tile has up to 32 rows of one adapter.  out = base + scale up (down x) is two products on
// the matrix cores, the small one in between never leaving the registers:
//
//   h [rank][rows]    = down [rank][k] x^T [k][rows]      (k long: its waves split it, LDS joins)
//   out^T [m][rows]   = up [m][rank] h [rank][rows]       (m long: its waves split it)
//
// With rows in the columns of both, a lane ends the first product with h at row l % 16 and
// ranks 4 (l / 16) + i, i < 4 (l its place in the wave), which is what it has to hand to the
// second, if the order of its terms is chosen so: no exchange between lanes.  16-bit weights
// take h as the sum of two bfloat16 (h to 2^-17 of itself; one alone would round it to 2^-9),
// in the two halves of one instruction's terms.  float16 weights are split alike for this
// product, since h may be past float16's range; their first product is in float16.
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

// The rows' h as terms of the second product: 4 ranks, in 16-bit types their two parts.
template <int W>
__device__ __forceinline__ Frag h_terms(f32x4 h)
{
    Frag f;
    if constexpr (W == kF32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f.w[i] = __float_as_uint(h[i]);
    } else {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            split(h[i], hi[i], lo[i]);
        f.w[0] = hi[0] | hi[1] << 16;
        f.w[1] = hi[2] | hi[3] << 16;
        f.w[2] = lo[0] | lo[1] << 16;
        f.w[3] = lo[2] | lo[3] << 16;
    }
    return f;
}

// c += w h for 4 ranks of w (two words of 16-bit weights, four of float32).
template <int W>
__device__ __forceinline__ f32x4 mma_h(const uint32_t (&w)[kSize<W>], Frag h, f32x4 c)
{
    if constexpr (W == kF32) {
        return mma_f32({w[0], w[1], w[2], w[3]}, h, c);
    } else if constexpr (W == kBf16) {
        return mma_bf16({w[0], w[1], w[0], w[1]}, h, c);
    } else {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint16_t bits = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
            split((float)__builtin_bit_cast(_Float16, bits), hi[i], lo[i]);
        }
        const uint32_t h0 = hi[0] | hi[1] << 16, h1 = hi[2] | hi[3] << 16;
        const uint32_t l0 = lo[0] | lo[1] << 16, l1 = lo[2] | lo[3] << 16;
        return mma_bf16({l0, l1, l0, l1}, h, mma_bf16({h0, h1, h0, h1}, h, c));
    }
}

// base and out of one row: out columns [m, m + kEls) from their sums, as many as there are.
template <int W>
struct Output {
    const char *base;                   // the row's, or NULL
    char *out;
    bool base_i32, there;
    float base_scale, scale;
    int32_t m;

    __device__ __forceinline__ Frag load_base(int32_t col) const
    {
        if (!base || !there)
            return {{0, 0, 0, 0}};
        return load_frag<W>(base + (int64_t)col * kSize<W>, m - col);
    }
    __device__ __forceinline__ void store(int32_t col, const float (&sum)[kEls<W>],
                                          const Frag &b) const
    {
        if (!there || col >= m)
            return;
        uint32_t bits[kEls<W>];
#pragma unroll
        for (int u = 0; u < kEls<W>; ++u) {
            float from;
            if constexpr (W == kF32)
                from = base_i32 ? (float)(int32_t)b.w[u] : __uint_as_float(b.w[u]);
            else if constexpr (W == kBf16)
                from = __uint_as_float(u & 1 ? b.w[u / 2] & 0xFFFF0000u : b.w[u / 2] << 16);
            else
                from = (float)__builtin_bit_cast(_Float16,
                                                 (uint16_t)(b.w[u / 2] >> (16 * (u & 1))));
            bits[u] = el_bits<W>(base_scale * from + scale * sum[u]);
        }
        char *to = out + (int64_t)col * kSize<W>;
        if (col + kEls<W> <= m) {
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

// NW waves a tile (1: a block has four tiles, each wave its own), 16 RT rows of it, 16 CT
// ranks.
template <int W, int X, int CT, int RT, int NW, bool BACK>
__global__ __launch_bounds__(NW == 1 ? 256 : NW * kWave) void k_pass(PassArgs a)
{
    constexpr int E = kEls<W>, S = kSize<W>, kUnit = 2 * 4 * E;   // terms of 128 bytes of a row
    constexpr int kAcc = CT * RT * 4;
    __shared__ float joined[NW > 1 ? NW * kAcc * kWave : 1];
    const int lane = threadIdx.x % kWave, col = lane % 16, quad = lane / 16;
    const int wave = NW > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave) : 0;
    int64_t tile = blockIdx.x / a.splits;
    const int split_at = (int)(blockIdx.x - tile * a.splits);
    if constexpr (NW == 1) {
        tile = tile * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
        if (tile >= a.n_tiles)
            return;
    }
    Piece4 p;
    if (a.tiles) {
        p = a.tiles[tile];
        if (p.group < 0)
            return;
    } else {
        const int32_t id = a.ids[tile];
        p = {id >= 0 && id < a.groups ? id : a.groups, (int32_t)tile, 1, 0};
    }
    int32_t row[RT];
    bool there[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int32_t at = rt * 16 + col;
        there[rt] = at < p.count;
        const int32_t place = p.first + (there[rt] ? at : 0);
        row[rt] = a.order ? a.order[place] : place;
    }
    const bool adapted = p.group < a.groups;
    f32x4 h[RT][CT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
            h[rt][ct] = f32x4{0, 0, 0, 0};
    if (adapted) {
        // ---- h = w1 x ----
        const char *x[RT], *w1[CT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
            x[rt] = a.x + row[rt] * a.x_stride;
        const char *first = a.w1 + p.group * a.w1_step;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            // ranks behind the last one read its weights: what comes of it is cleared below
            const int32_t r = min(ct * 16 + col, a.rank - 1);
            w1[ct] = first + (BACK ? (int64_t)r : (int64_t)r * a.k) * S;
        }
        const auto load_w1 = [&](int ct, int32_t k, int32_t left) __attribute__((always_inline)) {
            if constexpr (!BACK) {
                return load_frag<W>(w1[ct] + (int64_t)k * S, left);
            } else {
                Frag f;
                const char *at = w1[ct] + (int64_t)k * a.rank * S;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    f.w[i] = 0;
#pragma unroll
                for (int u = 0; u < E; ++u)
                    if (u < left) {
                        const char *el = at + (int64_t)u * a.rank * S;
                        if constexpr (S == 4)
                            f.w[u] = *reinterpret_cast<const uint32_t *>(el);
                        else
                            f.w[u / 2] |= (uint32_t)*reinterpret_cast<const uint16_t *>(el)
                                          << (16 * (u & 1));
                    }
                return f;
            }
        };
        const auto step = [&](int32_t k0, bool whole) __attribute__((always_inline)) {
            Frag fx[2][RT], fw[2][CT];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int32_t k = k0 + half * 4 * E + quad * E;
                const int32_t left = whole ? E : a.k - k;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    fx[half][rt] = load_frag<W>(x[rt] + (int64_t)k * S, left);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
                    fw[half][ct] = load_w1(ct, k, left);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const Frag t = to_terms<X>(fx[half][rt]);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
                        h[rt][ct] = mma<W>(fw[half][ct], t, h[rt][ct]);
                }
        };
        const int32_t whole = a.k / kUnit * kUnit;
        int32_t k0 = wave * kUnit;
#pragma unroll(CT <= 2 ? 2 : 1)
        for (; k0 < whole; k0 += NW * kUnit)
            step(k0, true);
        if (k0 < a.k)
            step(k0, false);
        // ---- the waves' parts, joined in order ----
        if constexpr (NW > 1) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        joined[(wave * kAcc + (rt * CT + ct) * 4 + i) * kWave + lane] =
                            h[rt][ct][i];
            __syncthreads();
            for (int e = threadIdx.x; e < kAcc * kWave; e += NW * kWave) {
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < NW; ++w)
                    sum += joined[w * kAcc * kWave + e];
                joined[e] = sum;                          // (only this lane reads or writes e)
            }
            __syncthreads();
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        h[rt][ct][i] = joined[((rt * CT + ct) * 4 + i) * kWave + lane];
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (ct * 16 + quad * 4 + i >= a.rank)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
                        h[rt][ct][i] = 0.0f;
    }
    if (a.hidden && split_at == 0 && wave == 0) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
            if (there[rt])
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int32_t r = ct * 16 + quad * 4 + i;
                        if (r < a.rank)
                            a.hidden[(int64_t)row[rt] * a.rank + r] = h[rt][ct][i];
                    }
    }
    if (!a.out)
        return;
    // ---- out = base + scale w2 h ----
    Output<W> o[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        o[rt].base = a.base ? a.base + row[rt] * a.base_stride : nullptr;
        o[rt].out = a.out + row[rt] * a.out_stride;
        o[rt].base_i32 = a.base_i32;
        o[rt].there = there[rt];
        o[rt].base_scale = a.base_scale;
        o[rt].scale = !adapted ? 0.0f : a.scales ? a.scales[p.group] : a.scale;
        o[rt].m = a.m;
    }
    Frag terms[RT][CT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
            terms[rt][ct] = h_terms<W>(h[rt][ct]);
    const char *w2 = a.w2 + (adapted ? p.group * a.w2_step : 0);
    if constexpr (!BACK) {
        // a unit: two tiles of 16 columns.  16-bit types give a lane 8 neighbours of them.
        constexpr int kCols = 32;
        const bool fours = a.rank % 4 == 0;
        const auto column = [&](int t, int place) __attribute__((always_inline)) {
            return S == 2 ? place / 4 * 8 + t * 4 + place % 4 : t * 16 + place;
        };
        for (int32_t m0 = (split_at * NW + wave) * kCols; m0 < a.m;
             m0 += a.splits * NW * kCols) {
            constexpr int kPieces = S == 2 ? 1 : 2;
            Frag b[RT][kPieces];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < kPieces; ++i)
                    b[rt][i] = o[rt].load_base(m0 + i * 16 + quad * E);
            f32x4 sum[2][RT];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    sum[t][rt] = f32x4{0, 0, 0, 0};
            if (adapted)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int32_t m = min(m0 + column(t, col), a.m - 1);
                    const char *from = w2 + (int64_t)m * a.rank * S;
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        const int32_t r = ct * 16 + quad * 4;
                        uint32_t w[S] = {};
                        if (fours) {
                            if (r < a.rank)
                                __builtin_memcpy(w, from + r * S, 4 * S);
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (r + i < a.rank) {
                                    if constexpr (S == 4)
                                        w[i] = reinterpret_cast<const uint32_t *>(from)[r + i];
                                    else
                                        w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(
                                                        from)[r + i] << (16 * (i & 1));
                                }
                        }
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt)
                            sum[t][rt] = mma_h<W>(w, terms[rt][ct], sum[t][rt]);
                    }
                }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    float v[E];
#pragma unroll
                    for (int u = 0; u < E; ++u)
                        v[u] = sum[S == 2 ? u / 4 : i][rt][u % 4];
                    o[rt].store(m0 + i * 16 + quad * E, v, b[rt][i]);
                }
        }
    } else {
        // a unit: E tiles of 16 columns; tile t has columns t, E + t, 2 E + t, ...
        constexpr int kCols = 16 * E;
        for (int32_t m0 = (split_at * NW + wave) * kCols; m0 < a.m;
             m0 += a.splits * NW * kCols) {
            f32x4 sum[E][RT];
#pragma unroll
            for (int t = 0; t < E; ++t)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    sum[t][rt] = f32x4{0, 0, 0, 0};
            if (adapted)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    Frag f[4];                            // 4 ranks of E columns
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int32_t r = ct * 16 + quad * 4 + i, m = m0 + col * E;
                        f[i] = load_frag<W>(w2 + ((int64_t)min(r, a.rank - 1) * a.m + m) * S,
                                            r < a.rank ? a.m - m : 0);
                    }
#pragma unroll
                    for (int t = 0; t < E; ++t) {
                        uint32_t w[S];
                        if constexpr (S == 4) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                w[i] = f[i].w[t];
                        } else {
                            constexpr uint32_t kLow = 0x05040100u, kHigh = 0x07060302u;
                            const uint32_t pick = t & 1 ? kHigh : kLow;
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                w[i] = __builtin_amdgcn_perm(f[2 * i + 1].w[t / 2],
                                                             f[2 * i].w[t / 2], pick);
                        }
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt)
                            sum[t][rt] = mma_h<W>(w, terms[rt][ct], sum[t][rt]);
                    }
                }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[E];
#pragma unroll
                    for (int t = 0; t < E; ++t)
                        v[t] = sum[t][rt][i];
                    const int32_t at = m0 + (quad * 4 + i) * E;
                    o[rt].store(at, v, o[rt].load_base(at));
                }
        }
    }
}

template <int W, int X, int CT, bool BACK>
hipError_t pass_of(const PassArgs &a, hipStream_t stream)
{
    // one wave a tile where a tile's two products are a few units of 128 bytes each
    constexpr int kNarrow = 8 * 128 / kSize<W>;
    constexpr int NW = CT > 2 ? 4 : 8;
    PassArgs b = a;
    b.splits = 1;
    if (a.tiles && a.k <= kNarrow && a.m <= kNarrow) {
        hipLaunchKernelGGL((k_pass<W, X, CT, 2, 1, BACK>), dim3((uint32_t)((a.n_tiles + 3) / 4)),
                           dim3(256), 0, stream, b);
        return hipGetLastError();
    }
    // few tiles: several blocks a tile, which share its columns (and all take its h)
    const int64_t most = (a.m + 128 * NW - 1) / (128 * NW);
    b.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(most, 512 / a.n_tiles));
    const dim3 grid((uint32_t)(a.n_tiles * b.splits));
    if (a.tiles)
        hipLaunchKernelGGL((k_pass<W, X, CT, 2, NW, BACK>), grid, dim3(NW * kWave), 0, stream, b);
    else
        hipLaunchKernelGGL((k_pass<W, X, CT, 1, NW, BACK>), grid, dim3(NW * kWave), 0, stream, b);
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
// D [rank][cols] = sum over a chunk's rows of h[row][rank] y[row][col]: a wave has 16 E
// columns, 32 rows (16 in float32) a step; a lane loads E columns of 8 (4) rows and turns
// them by byte permutes into the terms of E products, whose columns are t, E + t, ...
// h and, where they are no bfloat16, y are taken as sums of two bfloat16, as above.

template <int W, int CT>
__global__ __launch_bounds__(256) void k_grads(GradArgs a)
{
    constexpr int E = kEls<W>, S = kSize<W>, kRows = S == 4 ? 4 : 8;   // rows a lane and step
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
    const int32_t c0 = (block * 4 + wave) * 16 * E;
    if (c0 >= j.cols)
        return;
    const int32_t at = c0 + col * E, left = max(j.cols - at, 0);
    f32x4 sum[CT][E];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int t = 0; t < E; ++t)
            sum[ct][t] = f32x4{0, 0, 0, 0};
    const char *y = j.y + (left > 0 ? (int64_t)at * S : 0);
    for (int32_t s = 0; s < p.count; s += 4 * kRows) {
        Frag f[kRows];
        float hv[CT][kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int32_t place = s + quad * kRows + u;
            const bool there = place < p.count;
            const int64_t row = a.order[p.first + (there ? place : 0)];
            f[u] = load_frag<W>(y + row * j.y_stride, there ? left : 0);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const int32_t r = ct * 16 + col;
                hv[ct][u] = there && r < a.rank ? j.h[row * a.rank + r] : 0.0f;
            }
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
    // a group of one chunk is done; others leave a part of the sum
    const bool whole = a.chunk_starts[p.group + 1] - a.chunk_starts[p.group] == 1;
    const float scale = a.scales ? a.scales[p.group] : a.scale;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t r = ct * 16 + quad * 4 + i;
            if (r >= a.rank)
                continue;
#pragma unroll
            for (int t = 0; t < E; ++t) {
                if (t >= left)
                    continue;
                const float v = sum[ct][t][i];
                if (!whole) {
                    j.partial[((int64_t)p.slot * a.rank + r) * j.cols + at + t] = v;
                } else {
                    const int64_t to = (int64_t)p.group * a.rank * j.cols +
                                       (j.transposed ? (int64_t)(at + t) * a.rank + r
                                                     : (int64_t)r * j.cols + at + t);
                    if constexpr (S == 4)
                        reinterpret_cast<uint32_t *>(j.out)[to] = el_bits<W>(scale * v);
                    else
                        reinterpret_cast<uint16_t *>(j.out)[to] = (uint16_t)el_bits<W>(scale * v);
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
    const int32_t per_group = (int32_t)std::min<int64_t>(64, (els + 1023) / 1024);
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
    return 4 * 16 * kEls<W>;
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
