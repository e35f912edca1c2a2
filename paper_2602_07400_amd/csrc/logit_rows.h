// Rows of class scores or logits (internal): element types, a group of lanes that
// holds a row, reductions over the group and the order of a row's classes.
//
// A row of n classes belongs to a group of G lanes: part of a wave, a wave, or a
// block of several waves.  Lane t holds elements (j * G + t) * VEC + u, u < VEC,
// j < NV, in registers: one element a load for short rows, 16 bytes a load for
// long ones (at any alignment: rows of odd lengths start anywhere).  Rows longer
// than the registers hold are read again for every pass.
//
// The order of a row is descending logit, then ascending class.  A NaN, a -inf or
// (int32) the lowest integer is masked and has no place in it.  Selection works on
// 32-bit keys that grow with the logit; -0 and +0 have one key.
#pragma once

#include <type_traits>

#include "bl_internal.h"

namespace bl {
namespace rows {

constexpr int32_t kMaxClasses = 1 << 30;

enum : int { kI32 = 0, kF32 = 1, kF16 = 2, kBf16 = 3 };

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// f(integral_constant 0), ..., f(integral_constant N - 1): indexes of registers that are
// constants before any loop is unrolled.
template <int N, int I = 0, class F>
__device__ __forceinline__ void static_for(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        static_for<N, I + 1>(f);
    }
}

// ---- element types ----
// Cmp: what elements are compared as; kShift: key bits below the type's own.  minus: a
// difference v - from, v <= from, as float; -inf for a masked v.
template <int TYPE>
struct Elem {
    typedef float Cmp;
    static constexpr int kBytes = TYPE == kF32 ? 4 : 2;
    static constexpr int kShift = TYPE == kF32 ? 0 : TYPE == kF16 ? 13 : 16;
    static __device__ __forceinline__ Cmp lowest() { return -__builtin_inff(); }
    static __device__ __forceinline__ float to_float(Cmp v) { return v; }
    static __device__ __forceinline__ float minus(Cmp v, Cmp from) { return v - from; }
    static __device__ __forceinline__ uint32_t key(Cmp v)
    {
        const uint32_t b = __float_as_uint(v + 0.0f);
        return (b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) >> kShift;
    }
    // the element whose key is k (for a key that no element has: one between its neighbours)
    static __device__ __forceinline__ Cmp from_key(uint32_t k)
    {
        k <<= kShift;
        if (!(k & 0x80000000u))
            k |= (1u << kShift) - 1;
        return __uint_as_float(k ^ ((k & 0x80000000u) ? 0x80000000u : 0xFFFFFFFFu));
    }
    static constexpr uint32_t kFirstKey = 0x00800000u >> kShift;   // of the lowest finite value
};

template <>
struct Elem<kI32> {
    typedef int32_t Cmp;
    static constexpr int kBytes = 4;
    static constexpr int kShift = 0;
    static __device__ __forceinline__ Cmp lowest() { return INT32_MIN; }
    static __device__ __forceinline__ float to_float(Cmp v) { return (float)v; }
    // in integers first: scores past 2^24 (an int8 head's reach 10^9) are not floats
    static __device__ __forceinline__ float minus(Cmp v, Cmp from)
    {
        const float less = -(float)((uint32_t)from - (uint32_t)v);
        return v == INT32_MIN ? -__builtin_inff() : less;
    }
    static __device__ __forceinline__ uint32_t key(Cmp v) { return (uint32_t)v ^ 0x80000000u; }
    static __device__ __forceinline__ Cmp from_key(uint32_t k)
    {
        return (int32_t)(k ^ 0x80000000u);
    }
    static constexpr uint32_t kFirstKey = 1;
};

// One element from memory, as it is compared.
template <int TYPE>
__device__ __forceinline__ typename Elem<TYPE>::Cmp load_one(const char *row, int64_t i)
{
    if constexpr (TYPE == kI32)
        return reinterpret_cast<const int32_t *>(row)[i];
    else if constexpr (TYPE == kF32)
        return reinterpret_cast<const float *>(row)[i];
    else if constexpr (TYPE == kF16)
        return (float)reinterpret_cast<const _Float16 *>(row)[i];
    else
        return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(row)[i] << 16);
}

// An element of a type known at run time, as float (teacher lists).
__device__ __forceinline__ float load_float(const char *p, int type, int64_t i)
{
    switch (type) {
    case kI32: return (float)load_one<kI32>(p, i);
    case kF32: return load_one<kF32>(p, i);
    case kF16: return load_one<kF16>(p, i);
    default: return load_one<kBf16>(p, i);
    }
}

// ---- pieces: VEC elements in registers ----
template <int TYPE, int VEC>
struct Piece {
    static constexpr int kWords = VEC * Elem<TYPE>::kBytes >= 4 ? VEC * Elem<TYPE>::kBytes / 4 : 1;
    uint32_t w[kWords];

    __device__ __forceinline__ typename Elem<TYPE>::Cmp get(int u) const
    {
        if constexpr (TYPE == kI32) {
            return (int32_t)w[u];
        } else if constexpr (TYPE == kF32) {
            return __uint_as_float(w[u]);
        } else if constexpr (TYPE == kBf16) {
            return __uint_as_float(u & 1 ? w[u / 2] & 0xFFFF0000u : w[u / 2] << 16);
        } else {
            f16x2 h;
            __builtin_memcpy(&h, &w[u / 2], 4);
            return (float)(u & 1 ? h[1] : h[0]);
        }
    }
    __device__ __forceinline__ void fill_masked()
    {
        constexpr uint32_t m = TYPE == kI32 ? 0x80000000u : TYPE == kF32 ? 0xFF800000u
                               : TYPE == kF16 ? 0xFC00FC00u : 0xFF80FF80u;
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            w[i] = m;
    }
    // elements [first + i, first + i + VEC) of a row of n, `first` the same in the whole
    // wave (an address in scalar registers and a 32-bit offset); those past it are masked
    __device__ __forceinline__ void load(const char *row, int32_t first, int32_t i, int32_t n)
    {
        const char *p = row + (int64_t)first * Elem<TYPE>::kBytes + (uint32_t)(i * Elem<TYPE>::kBytes);
        i += first;
        if (i + VEC <= n) {
            if constexpr (VEC * Elem<TYPE>::kBytes >= 4) {
                __builtin_memcpy(w, p, sizeof w);
            } else {
                w[0] = *reinterpret_cast<const uint16_t *>(p);
            }
            return;
        }
        fill_masked();
        // the end of the row: from its last element on, each pushes the ones behind it up
        if constexpr (VEC > 1)
            for (int u = n - i - 1; u >= 0; --u) {
                if constexpr (Elem<TYPE>::kBytes == 4) {
#pragma unroll
                    for (int k = kWords - 1; k > 0; --k)
                        w[k] = w[k - 1];
                    w[0] = reinterpret_cast<const uint32_t *>(p)[u];
                } else {
#pragma unroll
                    for (int k = kWords - 1; k > 0; --k)
                        w[k] = __builtin_amdgcn_alignbit(w[k], w[k - 1], 16);
                    w[0] = w[0] << 16 | reinterpret_cast<const uint16_t *>(p)[u];
                }
            }
    }
    __device__ __forceinline__ void put16(int u, uint32_t v)
    {
        w[u / 2] = u & 1 ? (w[u / 2] & 0x0000FFFFu) | v << 16 : (w[u / 2] & 0xFFFF0000u) | v;
    }
    // element u (a run-time index) masked
    __device__ __forceinline__ void mask(int at)
    {
#pragma unroll
        for (int u = 0; u < VEC; ++u)
            if (u == at) {
                if constexpr (Elem<TYPE>::kBytes == 4)
                    w[u] = TYPE == kI32 ? 0x80000000u : 0xFF800000u;
                else
                    put16(u, TYPE == kF16 ? 0xFC00u : 0xFF80u);
            }
    }
};

// ---- reductions over the lanes of a group ----
// The value of the lane that holds the other half's result of a reduction over
// 2 S lanes, once every S lanes hold theirs: within a row of 16 lanes by DPP.
template <int S>
__device__ __forceinline__ uint32_t other_half(uint32_t v)
{
    constexpr int ctrl = S == 1 ? 0xB1 : S == 2 ? 0x4E : S == 4 ? 0x141 : 0x140;
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xF, 0xF, true);
}

template <int S, class T, class Op>
__device__ __forceinline__ T reduce_step(T v, Op op)
{
    static_assert(sizeof(T) == 4 || sizeof(T) == 8, "32- or 64-bit values");
    constexpr int W = sizeof(T) / 4;
    uint32_t a[W], x[W], y[W];
    __builtin_memcpy(a, &v, sizeof v);
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if constexpr (S <= 8) {
            x[i] = a[i];
            y[i] = other_half<S>(a[i]);
        } else if constexpr (S == 16) {
            const auto r = __builtin_amdgcn_permlane16_swap(a[i], a[i], false, false);
            x[i] = r[0];
            y[i] = r[1];
        } else {
            const auto r = __builtin_amdgcn_permlane32_swap(a[i], a[i], false, false);
            x[i] = r[0];
            y[i] = r[1];
        }
    }
    T p, q;
    __builtin_memcpy(&p, x, sizeof p);
    __builtin_memcpy(&q, y, sizeof q);
    return op(p, q);
}

// Over G <= 64 lanes of a wave; every lane gets the result.
template <int G, class T, class Op>
__device__ __forceinline__ T wave_reduce(T v, Op op)
{
    if constexpr (G > 1) v = reduce_step<1>(v, op);
    if constexpr (G > 2) v = reduce_step<2>(v, op);
    if constexpr (G > 4) v = reduce_step<4>(v, op);
    if constexpr (G > 8) v = reduce_step<8>(v, op);
    if constexpr (G > 16) v = reduce_step<16>(v, op);
    if constexpr (G > 32) v = reduce_step<32>(v, op);
    return v;
}

constexpr int kMaxWaves = 16;

// LDS of one group's reductions and scans (only groups of several waves use it).
struct Scratch {
    uint64_t slot[2][kMaxWaves];
};

struct Max {
    template <class T> __device__ T operator()(T a, T b) const { return a > b ? a : b; }
    // the other one where one is a NaN
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Add {
    template <class T> __device__ T operator()(T a, T b) const { return a + b; }
};

// A group of G lanes; t is the lane's place in it.  Reductions of several waves
// go through LDS, alternating between two sets of slots so that one barrier each
// is enough.
template <int G>
struct Group {
    int t;
    Scratch *s;
    int turn;

    __device__ __forceinline__ Group(int place, Scratch *scratch) : t(place), s(scratch), turn(0) {}

    __device__ __forceinline__ void barrier()
    {
        if constexpr (G > kWave) {
            __syncthreads();
        } else {
            // one wave: LDS accesses run in order; keep the compiler's order too
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }

    template <class T, class Op>
    __device__ __forceinline__ T reduce(T v, Op op)
    {
        v = wave_reduce<(G < kWave ? G : kWave)>(v, op);
        if constexpr (G > kWave) {
            constexpr int W = G / kWave;
            T *slot = reinterpret_cast<T *>(s->slot[turn]);
            turn ^= 1;
            if (t % kWave == 0)
                slot[t / kWave] = v;
            __syncthreads();
            v = wave_reduce<W>(slot[t % W], op);
        }
        return v;
    }

    // the sum of v over the lanes before this one, and (total) over all
    template <class T>
    __device__ __forceinline__ T scan(T v, T &total)
    {
        constexpr int L = G < kWave ? G : kWave;
        T in = v;
#pragma unroll
        for (int d = 1; d < L; d *= 2) {
            const T o = __shfl_up(in, d, L);
            if (t % L >= d)
                in += o;
        }
        total = __shfl(in, L - 1, L);
        T before = __shfl_up(in, 1, L);
        if (t % L == 0)
            before = 0;
        if constexpr (G > kWave) {
            constexpr int W = G / kWave;
            T *slot = reinterpret_cast<T *>(s->slot[turn]);
            turn ^= 1;
            if (t % kWave == 0)
                slot[t / kWave] = total;
            __syncthreads();
            total = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const T c = slot[w];
                if (w < t / kWave)
                    before += c;
                total += c;
            }
        }
        return before;
    }
};

// ---- a row in a group's registers, or in memory ----
// KEEP: the pieces stay in registers from pass to pass.  Without, a row is read once by
// each(), kBatch pieces at a time: half the registers, twice the blocks on a CU.
template <int TYPE, int G, int NV, int VEC, bool RESIDENT, bool KEEP = true>
struct Row {
    typedef typename Elem<TYPE>::Cmp Cmp;
    typedef Piece<TYPE, VEC> P;
    static constexpr int kSpan = G * VEC;                 // elements of one piece per lane
    static constexpr int kFlight = 4;                     // pieces that stream() loads together
    const char *row;
    int32_t n, t;
    static constexpr int kBatch = NV < 8 ? NV : 8;
    P piece[RESIDENT && KEEP ? NV : 1];

    __device__ __forceinline__ Row(const char *r, int32_t classes, int lane)
        : row(r), n(classes), t(lane)
    {
        if constexpr (RESIDENT && KEEP) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (j * kSpan < n)
                    piece[j].load(row, j * kSpan, t * VEC, n);
                else
                    piece[j].fill_masked();
            }
        }
    }

    // f(j, its first element, piece j) in index order of the pieces; j is an
    // integral_constant where the row is in registers
    template <class F>
    __device__ __forceinline__ void each(F f)
    {
        if constexpr (RESIDENT && !KEEP)
            static_for<NV / kBatch>([&](auto B) __attribute__((always_inline)) {
                constexpr int j0 = decltype(B)::value * kBatch;
                if (j0 * kSpan >= n)
                    return;
                P p[kBatch];
                static_for<kBatch>([&](auto j) __attribute__((always_inline)) {
                    p[j].load(row, (j0 + j) * kSpan, t * VEC, n);
                });
                static_for<kBatch>([&](auto j) __attribute__((always_inline)) {
                    f(std::integral_constant<int, j0 + decltype(j)::value>(),
                      (j0 + j) * kSpan + t * VEC, p[j]);
                });
            });
        else if constexpr (RESIDENT)
            static_for<NV>([&](auto J) __attribute__((always_inline)) {
                constexpr int j = decltype(J)::value;
                if (j * kSpan < n) {
                    again<j>();
                    f(J, j * kSpan + t * VEC, piece[j]);
                }
            });
        else
            stream<kFlight>([&](int32_t i, const P &p) __attribute__((always_inline)) {
                f(i / kSpan, i, p);
            });
    }

    // Piece j to be unpacked again: kept unpacked from an earlier pass, the elements
    // would take more registers than there are.
    template <int j>
    __device__ __forceinline__ void again()
    {
        if constexpr (VEC > 1)
#pragma unroll
            for (int i = 0; i < P::kWords; ++i)
                asm("" : "+v"(piece[j].w[i]));
    }

    // f(first element, piece) for all pieces, read again from memory in a loop: for what is
    // seldom done.  Unrolled over the registers it makes long code that takes registers
    // from what is done always (plain draws of 1024 x 50021: 88 -> 190 us with spills).
    // hits: one bit a piece of the lane, from the first on; pieces without one in any lane
    // of a wave may be left out.
    template <int FLIGHT = kFlight, class F>
    __device__ __forceinline__ void stream(F f, uint32_t hits = 0xFFFFFFFFu) const
    {
        for (int32_t i = 0; i < n; i += FLIGHT * kSpan) {
            if constexpr (RESIDENT) {
                const bool any = __any(hits & ((1u << FLIGHT) - 1));
                hits >>= FLIGHT;
                if (!any)
                    continue;
            }
            P p[FLIGHT];
            static_for<FLIGHT>([&](auto j) __attribute__((always_inline)) {
                p[j].load(row, i + j * kSpan, t * VEC, n);
            });
            static_for<FLIGHT>([&](auto j) __attribute__((always_inline)) {
                f(i + j * kSpan + t * VEC, p[j]);
            });
        }
    }
};

// 1 / T, and for a T below the normal numbers, where that may be no float, 2^126.
__host__ __device__ __forceinline__ float inverse(float temperature)
{
    return fminf(1.0f / temperature, 0x1p126f);
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// e^x, x <= 0, by the hardware's exponential of base 2: the roundings of the product and of
// log2(e) are an error of at most 1.3 |x| 2^-24 of the result, below 1e-6 of a weight that
// is 1e-5 of the largest.  (1 / T is rounded too, as in any 32-bit form that multiplies
// by it: |x| 2^-24.)
__device__ __forceinline__ float exp_fast(float x)
{
    return __builtin_amdgcn_exp2f(x * kLog2e);
}

// A lane's sum s of a row's terms, a piece at a time: part = start(), the piece's terms
// added to it, add(part).  LONG (a row in memory, any number of pieces): a piece's own sum
// goes to the total together with what the total's last rounding lost.  Added one by one,
// equal terms round the same way: over 2^24 classes, 2^14 a lane, 1.2e-4 of the sum.
template <bool LONG>
struct Total {
    float s = 0.0f, lost = 0.0f;
    __device__ __forceinline__ float start() const { return LONG ? 0.0f : s; }
    __device__ __forceinline__ void add(float part)
    {
        if constexpr (LONG) {
            const float more = part + lost, to = s + more;
            lost = more - (to - s);
            s = to;
        } else {
            s = part;
        }
    }
};

// A running maximum m of z and the sum s of 2^(c (z - m)): with c = log2(e) / T the
// exponentials of a softmax at temperature T.  The difference comes first: c z alone
// overflows where z is its type's lowest value, which masks are made of.  c is a product
// rounded once: the errors are those of exp_fast and |z - m| / T 2^-24 more.
template <int TYPE, bool LONG = false>
struct Softmax : Total<LONG> {
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    using Total<LONG>::s;
    using Total<LONG>::lost;
    Cmp m = E::lowest();
    __device__ __forceinline__ Cmp from() const
    {
        return TYPE != kI32 && m == E::lowest() ? 0 : m;
    }
    __device__ __forceinline__ void raise(Cmp to, float c)
    {
        const Cmp old = from();
        m = Max()(m, to);
        const float f = __builtin_amdgcn_exp2f(s == 0.0f ? 0.0f : E::minus(old, from()) * c);
        s *= f;
        if constexpr (LONG)
            lost *= f;
    }
    // log sum e^(z / T); the hardware's log2 times ln 2 has two roundings of log s
    __device__ __forceinline__ float log_norm(float inv_t) const
    {
        if (m == E::lowest())
            return -__builtin_inff();
        const float most = E::to_float(m);
        return most == __builtin_inff() ? most
                                        : most * inv_t + __builtin_amdgcn_logf(s) * kLn2;
    }
};

// Over a group: the maximum first, then the sums relative to it.
template <class Grp, int TYPE, bool LONG>
__device__ __forceinline__ Softmax<TYPE, LONG> combine(Grp &g, Softmax<TYPE, LONG> a, float c)
{
    a.raise(g.reduce(a.m, Max()), c);
    a.s = g.reduce(a.s, Add());
    return a;
}

// A value that all lanes of a wave have, in scalar registers.
template <class T>
__device__ __forceinline__ T uniform(T v)
{
    int w[sizeof(T) / 4];
    __builtin_memcpy(w, &v, sizeof v);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 4; ++i)
        w[i] = __builtin_amdgcn_readfirstlane(w[i]);
    __builtin_memcpy(&v, w, sizeof v);
    return v;
}

// ---- lists of candidates ----
// An element with its place in the order: larger entries come first.
__device__ __forceinline__ uint64_t entry(uint32_t key, int32_t cls)
{
    return (uint64_t)key << 32 | ~(uint32_t)cls;
}
__device__ __forceinline__ int32_t class_of(uint64_t e) { return (int32_t)~(uint32_t)e; }
__device__ __forceinline__ uint32_t key_of(uint64_t e) { return (uint32_t)(e >> 32); }

// A key that at least m of the group's G keys (one a lane, 1 <= m <= G) reach: the
// m-th largest, or a little less where that ends the search early.  room: G words of
// LDS.  A group of several waves leaves the search to its first one.
template <int G>
__device__ __forceinline__ uint32_t group_mth(Group<G> &g, uint32_t key, uint32_t m,
                                              uint32_t *room)
{
    constexpr int N = G / kWave;
    uint32_t lo = 0;
    if constexpr (N > 1) {
        room[g.t] = key;
        g.barrier();
    }
    if (g.t < kWave) {
        uint32_t keys[N], hi = 0, no = 0;                 // no: ~ the least
#pragma unroll
        for (int i = 0; i < N; ++i) {
            keys[i] = N > 1 ? room[i * kWave + g.t] : key;
            hi = max(hi, keys[i]);
            no = max(no, ~keys[i]);
        }
        hi = wave_reduce<kWave>(hi, Max());
        lo = ~wave_reduce<kWave>(no, Max());
        while (hi - lo > 1) {                             // count(>= lo) >= m
            const uint32_t mid = lo + (hi - lo) / 2;
            uint32_t count = 0;
#pragma unroll
            for (int i = 0; i < N; ++i)
                count += __popcll(__ballot(keys[i] >= mid));
            if (count >= m)
                lo = mid;
            else
                hi = mid;
            if (count >= m && count <= m + m / 8)
                break;
        }
    }
    if constexpr (N > 1) {
        g.barrier();
        if (g.t == 0)
            room[0] = lo;
        g.barrier();
        lo = room[0];
    }
    return lo;
}

// The lane's pieces whose largest logits reach `at`, as a bit each.
template <class L, class Cmp>
__device__ __forceinline__ uint32_t pieces_from(const Cmp (&most)[L::NV], Cmp at)
{
    uint32_t hits = 0xFFFFFFFFu;
    if constexpr (L::RESIDENT) {
        hits = 0;
        static_for<L::NV>([&](auto j) __attribute__((always_inline)) {
            hits |= (uint32_t)(most[j] >= at) << j;
        });
    }
    return hits;
}

// Appends the row's entries with lo <= logit to a list in LDS (fill: its length,
// cleared here), as many as it holds, and returns their number.  most: the largest
// logit of each of the lane's pieces; a piece that has candidates is loaded again, in
// a loop, since 16 pieces' unrolled searches take longer to fetch than to run.
template <int TYPE, class L, class R>
__device__ __forceinline__ uint32_t collect(Group<L::G> &g, R &row,
                                            const typename Elem<TYPE>::Cmp (&most)[L::NV],
                                            typename Elem<TYPE>::Cmp lo, uint64_t *list,
                                            uint32_t *fill)
{
    typedef Elem<TYPE> E;
    const auto search = [&](int32_t i, const Piece<TYPE, L::VEC> &p) __attribute__((always_inline)) {
        uint32_t in = 0;
#pragma unroll
        for (int u = 0; u < L::VEC; ++u)
            in |= (uint32_t)(p.get(u) >= lo) << u;
        if (!in)
            return;
        uint32_t to = atomicAdd(fill, __builtin_popcount(in));
#pragma unroll
        for (int u = 0; u < L::VEC; ++u)
            if (in >> u & 1) {
                if (to < (uint32_t)L::kList)
                    list[to] = entry(E::key(p.get(u)), i + u);
                ++to;
            }
    };
    g.barrier();
    if (g.t == 0)
        *fill = 0;
    g.barrier();
    if constexpr (L::RESIDENT) {
        uint32_t hits = pieces_from<L>(most, lo);
        while (hits) {
            const int j = __builtin_ctz(hits);
            hits &= hits - 1;
            const int32_t i = (j * L::G + g.t) * L::VEC;
            Piece<TYPE, L::VEC> p;
            p.load(row.row, 0, i, row.n);
            search(i, p);
        }
    } else {
        row.stream([&](int32_t i, const Piece<TYPE, L::VEC> &p) { search(i, p); });
    }
    g.barrier();
    return *fill;
}

// A mass in fixed point: the low 52 bits.  to_mass leaves a double's exponent above them,
// which sums carry along until kMassBits takes it off: two instructions instead of the
// seven of a conversion to 64-bit integers.  In 32 bits a class's share of the mass of n
// would be rounded by up to n / 2^32 of itself, the same way wherever logits are equal:
// 1e-5 of the sum at 2^17 classes, 1e-3 at 2^24.
typedef unsigned long long Mass;
constexpr Mass kMassBits = (1ull << 52) - 1;
__device__ __forceinline__ Mass to_mass(float w, double unit)
{
    return (Mass)__double_as_longlong(__builtin_fma((double)w, unit, 0x1p52));
}

// Keys [lo, hi) of a block's row in which the sum of `weight` over the order reaches
// `goal` (>= 1), the sum before them and their own (for masses kUnknown: not yet summed,
// and 0: the goal is above the whole sum, which is `before`).
template <class Sum>
struct Range {
    uint32_t lo, hi;
    Sum before, here;
};
constexpr Mass kUnknown = ~0ull;

// Narrows a range to the one key that reaches the goal, or until everything down to its
// end sums to `enough`: the row's elements are summed in kBins intervals of equal width
// (in fixed point: their order does not matter), again in the interval that reaches the
// goal, and so on.  A level takes a factor of kBins off the range.  Sum: Mass, or uint32_t
// for numbers of classes, which are known beforehand to reach the goal (what else it takes
// costs registers: top 64 of 2048 x 131072 in bfloat16 125 us instead of 105).
// kCopies interleaved counters an interval, one for every eighth or fourth lane: many
// elements fall in few intervals (16-bit logits near -10 have 16 values a unit), and equal
// addresses take turns.  bins: kBins * kCopies sums, in the memory of the list.  Masses by 8
// copies, and by 4 with twice the intervals: draws from 256 x 131072 (1024 lanes a row) 89.7
// and 91.5 us, from 108418 x 1051 (256 lanes) 1904 and 1846.
template <int TYPE, class L, class Sum, class R, class W>
__device__ __forceinline__ Range<Sum> narrow(Group<L::G> &g, R &row,
                                             const typename Elem<TYPE>::Cmp (&most)[L::NV],
                                             Range<Sum> in, Sum goal, Sum enough, Sum *bins,
                                             W weight)
{
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    constexpr bool kMass = sizeof(Sum) == 8;
    constexpr uint32_t kCopies = kMass && L::G == 256 ? 4 : 8;
    constexpr uint32_t kBins = L::kList * sizeof(uint64_t) / sizeof(Sum) / kCopies;
    constexpr uint32_t kRun = kBins > (uint32_t)L::G ? kBins / L::G : 1;
    const uint32_t copy = g.t % kCopies;
    bool by_key = TYPE == kI32;
    // No element has the key of -0 (+0's is the next one): as an end of the range it
    // would stand for +0, which may be outside.
    constexpr uint32_t kMinusZero = TYPE == kI32 ? 0xFFFFFFFFu : 0x7FFFFFFFu >> E::kShift;
    const auto off_minus_zero = [&]() __attribute__((always_inline)) {
        if constexpr (TYPE != kI32) {
            in.lo += in.lo == kMinusZero;
            in.hi -= in.hi == kMinusZero + 1;
        }
    };
    off_minus_zero();
    while ((in.hi - in.lo > 1 || (kMass && in.here == kUnknown)) &&
           in.before + in.here > enough) {
        // Floats by value, which crosses zero evenly, until that takes less than 15 of 16
        // keys off the range (an infinity or denormals at its end); integers, exactly, by
        // key, which takes kBins / 2 - 1 of kBins / 2 off at every level.
        const Cmp first = E::from_key(in.lo), last = E::from_key(in.hi - 1);
        uint32_t shift = 0;
        while ((in.hi - 1 - in.lo) >> shift >= kBins)
            ++shift;
        // half of each end, so that their difference does not overflow
        const float scale = (0.5f * (float)kBins) /
                            (0.5f * E::to_float(last) - 0.5f * E::to_float(first));
        const auto bin_of = [&](Cmp v) __attribute__((always_inline)) {
            const uint32_t b = by_key ? (in.hi - 1 - E::key(v)) >> shift
                                      : (uint32_t)((E::to_float(last) - E::to_float(v)) * scale);
            return min(b, kBins - 1);
        };
        g.barrier();
        for (uint32_t b = g.t; b < kBins * kCopies; b += L::G)
            bins[b] = 0;
        g.barrier();
        row.stream([&](int32_t, const Piece<TYPE, L::VEC> &p) {
#pragma unroll
            for (int u = 0; u < L::VEC; ++u) {
                const Cmp v = p.get(u);
                if (v >= first && v <= last)
                    atomicAdd(&bins[bin_of(v) * kCopies + copy], weight(v));
            }
        }, pieces_from<L>(most, first));
        g.barrier();
        const auto sum_of = [&](uint32_t b) __attribute__((always_inline)) {
            Sum sum = 0;
            for (uint32_t c = 0; c < kCopies; ++c) {
                const Sum own = b < kBins ? bins[b * kCopies + c] : 0;
                sum += kMass ? own & (Sum)kMassBits : own;
            }
            return sum;
        };
        Sum part = 0, total;
        for (uint32_t b = 0; b < kRun; ++b)
            part += sum_of(g.t * kRun + b);
        Sum before = in.before + g.scan(part, total), here = 0, base = 0;
        uint32_t found = 0;
        for (uint32_t b = 0; b < kRun; ++b) {
            const Sum own = kMass ? part : sum_of(g.t * kRun + b);
            if (before < goal && before + own >= goal) {
                found = g.t * kRun + b + 1;
                base = before;
                here = own;
            }
            before += own;
        }
        if constexpr (kMass) {
            // the lane that has it tells the others through the bins, which all have read
            static_assert(kRun == 1 && kBins >= 3, "an interval a lane");
            if (found) {
                bins[0] = found;
                bins[1] = base;
                bins[2] = here;
            }
            g.barrier();
            found = in.before + total >= goal ? (uint32_t)bins[0] : 0;
            base = bins[1];
            here = bins[2];
        } else {
            const uint64_t won = g.reduce((uint64_t)found << 32 | base, Max());
            found = (uint32_t)(won >> 32);
            base = (uint32_t)won;
            here = g.reduce(here, Max());
        }
        if (!found) {
            in = {in.lo, in.lo + 1, kMass ? in.before + total : goal, 0};
            break;
        }
        // the first key of the intervals up to `bound`, 64 keys at a time in every wave
        const auto first_key = [&](uint32_t bound) __attribute__((always_inline)) {
            uint32_t no = in.lo - 1, yes = in.hi - 1;
            while (yes - no > 1) {
                const uint64_t left = yes - no, step = (left - 1) / kWave + 1;
                const uint32_t ahead = (uint32_t)min(step * (g.t % kWave + 1), left);
                const uint64_t is = __ballot(bin_of(E::from_key(no + ahead)) < bound);
                const uint32_t at = __builtin_ctzll(is);  // (the last lane's is)
                yes = no + (uint32_t)min(step * (at + 1), left);
                no += (uint32_t)step * at;
            }
            return yes;
        };
        const uint32_t lo = first_key(found), hi = found == 1 ? in.hi : first_key(found - 1);
        by_key |= hi - lo > (in.hi - in.lo) / 16;
        in = {lo, hi, base, here};
        off_minus_zero();
        if constexpr (kMass)
            in = {uniform(in.lo), uniform(in.hi), uniform(in.before), uniform(in.here)};
    }
    return in;
}

// Sorting: each lane has EPL neighbouring entries in registers; exchanges within a
// lane and a wave need no barrier, only those between waves go through LDS.
template <int EPL, int G>
__device__ __forceinline__ void sort_runs(Group<G> &g, uint64_t *e, uint32_t p)
{
    constexpr uint32_t kInWave = (G < kWave ? G : kWave) * EPL;
    uint64_t x[EPL];
    const uint32_t first = g.t * EPL;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
        x[i] = first + i < p ? e[first + i] : 0;
    for (uint32_t size = 2; size <= p; size *= 2)
        for (uint32_t stride = size / 2; stride; stride /= 2) {
            uint64_t y[EPL];
            if (stride >= kInWave) {
                g.barrier();
#pragma unroll
                for (int i = 0; i < EPL; ++i)
                    if (first + i < p)
                        e[first + i] = x[i];
                g.barrier();
#pragma unroll
                for (int i = 0; i < EPL; ++i)
                    y[i] = first + i < p ? e[(first + i) ^ stride] : 0;
            } else if (stride >= EPL) {
#pragma unroll
                for (int i = 0; i < EPL; ++i)
                    y[i] = __shfl_xor(x[i], (int)(stride / EPL));
            } else {
#pragma unroll
                for (int d = 1; d < EPL; d *= 2)
                    if (stride == (uint32_t)d)
#pragma unroll
                        for (int i = 0; i < EPL; ++i)
                            y[i] = x[i ^ d];
            }
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                const uint32_t at = first + i;
                const bool larger = !(at & stride) == !(at & size);
                x[i] = (x[i] > y[i]) == larger ? x[i] : y[i];
            }
        }
    g.barrier();
#pragma unroll
    for (int i = 0; i < EPL; ++i)
        if (first + i < p)
            e[first + i] = x[i];
    g.barrier();
}

// c entries, at most 4 G of a block and 16 G of a wave, in descending order, in place;
// room for the next power of two.
template <int G>
__device__ __forceinline__ void sort_entries(Group<G> &g, uint64_t *e, uint32_t c)
{
    uint32_t p = 2;
    while (p < c)
        p *= 2;
    for (uint32_t i = c + g.t; i < p; i += G)
        e[i] = 0;
    g.barrier();
    if (p <= G)
        sort_runs<1>(g, e, p);
    else if (p <= 2 * G)
        sort_runs<2>(g, e, p);
    else if (G > kWave || p <= 4 * G)
        sort_runs<4>(g, e, p);
    else if constexpr (G <= kWave)
        sort_runs<16>(g, e, p);
}

// c entries in descending order to `to`: an entry's place is the number of larger
// ones, counted by G / (next power of two of c) neighbouring lanes.  f(entry) runs
// for every entry before the counting, and its result goes to with[place].
template <int G, class F>
__device__ __forceinline__ void place_entries(Group<G> &g, const uint64_t *e, uint32_t c,
                                              uint64_t *to, float *with, F f)
{
    uint32_t lanes = G;                                   // for an entry
    while (lanes > 1 && c * lanes > G)
        lanes /= 2;
    lanes = min(lanes, 16u);
    for (uint32_t base = 0; base < c; base += G / lanes) {
        const uint32_t at = base + g.t / lanes;
        const uint64_t mine = at < c ? e[at] : 0;
        float number = 0.0f;
        if (at < c && g.t % lanes == 0)
            number = f(mine);
        uint32_t place = 0;
        if (at < c)
            for (uint32_t i = g.t % lanes; i < c; i += lanes)
                place += e[i] > mine;
        for (uint32_t d = 1; d < lanes; d *= 2)
            place += __shfl_xor(place, (int)d);
        if (at < c && g.t % lanes == 0) {
            to[place] = mine;
            if (with)
                with[place] = number;
        }
    }
    g.barrier();
}

// The lane's group in its block, in a scalar register where a group is whole waves.
template <int G>
__device__ __forceinline__ int group_of()
{
    if constexpr (G >= 256)
        return 0;
    else if constexpr (G == kWave)
        return __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    else
        return threadIdx.x / G;
}

// ---- which group holds rows of n classes ----
template <int G_, int NV_, int VEC_, bool RESIDENT_>
struct Layout {
    static constexpr int G = G_, NV = NV_, VEC = VEC_;
    static constexpr bool RESIDENT = RESIDENT_;
    static constexpr int kSpan = G * VEC;                 // elements of one piece per lane
    static constexpr int kBlock = G < 256 ? 256 : G;
    static constexpr int kGroups = kBlock / G;            // rows of a block
    // Candidates of a row that LDS holds (a power of two; all the classes of a row
    // within a wave), and how many are put in order by counting rather than sorting:
    // c entries compare c^2 / G times a lane, 128 of them as long as a sort takes.
    static constexpr int kList = G >= 256 ? 4 * G : NV * VEC * G;
    static constexpr int kCounted =
        G == 1024 ? 352 : G == 512 ? 256 : G == 256 ? 176 : G == 64 ? 88 : NV * VEC * G;
    // waves a SIMD to compile for, where a row stays in registers
    static constexpr int kWavesPerSimd =
        !RESIDENT || G == kWave || NV * (VEC > 4 ? 4 : VEC) > 16 ? 4 : 8;
};

// f(Layout) for rows of n classes of a type whose lists have up to k entries a row.
template <int TYPE, class F>
hipError_t with_layout(int32_t n, int32_t k, F f)
{
    constexpr int V = 16 / Elem<TYPE>::kBytes;            // elements of a 16-byte load
    if (n <= 16 && k <= 16)
        return f(Layout<8, 2, 1, true>());
    if (n <= 64 && k <= 64)
        return f(Layout<16, 4, 1, true>());
    if (n <= 128 && k <= 128)
        return f(Layout<32, 4, 1, true>());
    if (n <= 512)
        return f(Layout<64, 8, 1, true>());
    if (n <= 1024)
        return f(Layout<64, 16 / V, V, true>());
    if (n <= 8192)
        return f(Layout<256, 32 / V, V, true>());
    if (n <= 512 * 8 * V)
        return f(Layout<512, 8, V, true>());
    if (n <= 1024 * 8 * V)
        return f(Layout<1024, 8, V, true>());
    if (n <= 1024 * 16 * V)
        return f(Layout<1024, 16, V, true>());
    return f(Layout<1024, 1, V, false>());
}

template <class F>
hipError_t with_type(int32_t type, F f)
{
    switch (type) {
    case kI32: return f(std::integral_constant<int, kI32>());
    case kF32: return f(std::integral_constant<int, kF32>());
    case kF16: return f(std::integral_constant<int, kF16>());
    default: return f(std::integral_constant<int, kBf16>());
    }
}

// launch(args, blocks) for all rows: a launch has fewer than 2^32 lanes, so that from 2^24
// rows of a block of 256 on it takes several.  args.skip(n) moves its pointers n rows on.
template <class Args, class F>
hipError_t in_launches(Args a, int block, int rows_a_block, F launch)
{
    const int64_t most = (((int64_t)1 << 32) / block - 1) * rows_a_block;
    hipError_t err = hipSuccess;
    for (int64_t left = a.n_rows; left > 0 && err == hipSuccess; left -= most) {
        a.n_rows = left < most ? left : most;
        launch(a, (uint32_t)((a.n_rows + rows_a_block - 1) / rows_a_block));
        err = hipGetLastError();
        a.skip(a.n_rows);
    }
    return err;
}

// ---- a lane a row: many short rows ----
// A wave takes 64 or 16 rows of up to kLaneClasses classes through a tile in LDS, and a
// lane or four go through a row: few reductions or none, and what is done once a row is
// done for many of them.  It pays once there are rows for all the GPU's waves: how many is
// at the kernels' launches.
constexpr int32_t kLaneClasses = 128;

// Orders a wave's LDS accesses: they run in order; the compiler keeps them so.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The rows' elements into the tile, as they are compared (32 bits).  Element e of the
// rows' n * rows is in row e / n = e * ceil(2^20 / n) >> 20: exact below 2^13, n <= 128.
template <int TYPE>
__device__ __forceinline__ void load_tile(const char *src, int64_t stride, int32_t rows,
                                          int32_t n, int32_t pitch, uint32_t *tile)
{
    typedef typename Elem<TYPE>::Cmp Cmp;
    constexpr int kFlight = 16;
    const uint32_t inverse = ((1u << 20) + n - 1) / n, count = (uint32_t)(rows * n);
    for (uint32_t e = threadIdx.x % kWave; e < count; e += kFlight * kWave) {
        Cmp v[kFlight];
        uint32_t to[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const uint32_t at = min(e + u * kWave, count - 1), r = at * inverse >> 20;
            const uint32_t col = at - r * n;
            to[u] = r * pitch + col;
            v[u] = load_one<TYPE>(src + r * stride, col);
        }
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (e + u * kWave < count)
                __builtin_memcpy(&tile[to[u]], &v[u], 4);
    }
}

}  // namespace rows
}  // namespace bl
