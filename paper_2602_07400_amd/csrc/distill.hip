// Distillation from a teacher's top logits, loss and gradient.
//
// A row has the student's logits z and a list J of distinct classes with the
// teacher's logits t.  With p = softmax(z / Ts), q_j = e^(t_j / Tt - log_norm) and a
// row weight w,
//
//   loss    = w [ sum_J q_j (log q_j - log p_j)  +  q_r (log q_r - log p_r) ]
//   dl/dz_i = w / Ts [ (Q + q_r) p_i - q_i ]               i in J
//           = w / Ts   (Q + q_r - q_r / p_r) p_i           elsewhere
//
// where Q = sum_J q_j.  With the teacher's log_norm given, the rest counts as one
// more class: q_r = max(0, 1 - Q), p_r = the student's mass outside J, summed over
// those classes themselves (1 - sum_J p_j would cancel).  Without it, log_norm is
// that of the list and q_r = 0.
//
// What bounds it: HBM with the gradient, 4096 x 65536 bf16, k 64: 215 us, 5.0 TB/s of
// the 5.8 of a plain copy, the VALU active in 75 of 100 cycles (an eighth of the rows has
// weight 0 and is written only); the loss alone, its exponentials (66 of 100) and the list
// in front of each row, 4099 x 32003 bf16: 65 us (92 with 1024 lanes that keep the row).
//
// The row is loaded once and stays in registers; the running maximum and sum of the
// softmax are taken as it arrives.  The list lies in LDS, linked per owning lane: a
// lane with entries masks them out of the sum over the rest and puts their gradient
// in its registers before it stores, so each gradient is stored once.
#include "logit_rows.h"

namespace bl {
namespace {

using namespace rows;

struct DistillArgs {
    const char *logits;
    int64_t stride;                     // bytes from row to row
    int64_t n_rows;
    int32_t n, k, top_type;
    float inv_t, inv_top_t;
    const char *top_values;             // [rows][k], top_type
    const int32_t *top_indices;         // [rows][k]
    const float *top_log_norm;          // [rows] or NULL
    const float *row_weight;            // [rows] or NULL
    float *loss;                        // [rows] or NULL
    char *grad;                         // or NULL, the logits' type
    int64_t grad_stride;                // bytes

    void skip(int64_t rows)
    {
        const auto on = [](auto *&p, int64_t by) { p = p ? p + by : p; };
        logits += rows * stride;
        top_values += rows * k * (top_type == kI32 || top_type == kF32 ? 4 : 2);
        top_indices += rows * k;
        on(top_log_norm, rows);
        on(row_weight, rows);
        on(loss, rows);
        on(grad, rows * grad_stride);
    }
};

// 2^(x log2(e) / T) = e^(x / T).  The factor in two parts: rounded to one, it would put
// the same relative error on every exponent, 7e-7 on the many classes at e^-10 of the
// largest, which a sum over them does not average out (one gradient can bear it).
// The second part is positive, so that -inf stays -inf: the smallest float at least, since
// hi itself comes down to 4e-39.
struct Scale {
    float hi, lo;
    __device__ __forceinline__ float left(float inv_t) const
    {
        return __builtin_fmaf(inv_t, kLog2e, -hi) + inv_t * 1.9259629e-8f;
    }
    __device__ __forceinline__ explicit Scale(float inv_t) : hi(inv_t * kLog2e)
    {
        if (!(left(inv_t) > 0.0f))
            hi = __uint_as_float(__float_as_uint(hi) - 1);
        lo = fmaxf(left(inv_t), 1.4e-45f);
    }
    __device__ __forceinline__ float pow(float x) const
    {
        return __builtin_amdgcn_exp2f(__builtin_fmaf(x, lo, x * hi));
    }
};

template <int TYPE, int VEC>
__device__ __forceinline__ void store_piece(char *row, int32_t first, int32_t i, int32_t n,
                                            const float (&v)[VEC])
{
    if constexpr (TYPE == kF32) {
        float *o = reinterpret_cast<float *>(row) + first + (uint32_t)i;
        i += first;
        if (i + VEC <= n) {
            __builtin_memcpy(o, v, sizeof v);
        } else if constexpr (VEC > 1) {                   // the end of the row
            float left[VEC];
            __builtin_memcpy(left, v, sizeof v);
            for (int u = 0; u < n - i; ++u) {
                o[u] = left[0];
#pragma unroll
                for (int k = 0; k < VEC - 1; ++k)
                    left[k] = left[k + 1];
            }
        }
    } else {
        typedef typename std::conditional<TYPE == kF16, _Float16, __bf16>::type H;
        H h[VEC];
        if constexpr (VEC == 1) {
            h[0] = (H)v[0];
        } else {
            typedef H H2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int u = 0; u < VEC; u += 2) {
                const H2 two = __builtin_convertvector((f32x2){v[u], v[u + 1]}, H2);
                h[u] = two[0];
                h[u + 1] = two[1];
            }
        }
        H *o = reinterpret_cast<H *>(row) + first + (uint32_t)i;
        i += first;
        if (i + VEC <= n) {
            __builtin_memcpy(o, h, sizeof h);
        } else if constexpr (VEC > 1) {
            uint32_t left[VEC / 2];
            __builtin_memcpy(left, h, sizeof h);
            for (int u = 0; u < n - i; ++u) {
                reinterpret_cast<uint16_t *>(o)[u] = (uint16_t)left[0];
#pragma unroll
                for (int k = 0; k < VEC / 2 - 1; ++k)
                    left[k] = __builtin_amdgcn_alignbit(left[k + 1], left[k], 16);
                left[VEC / 2 - 1] >>= 16;
            }
        }
    }
}

// A teacher's entry in LDS.
template <class Cmp>
struct Entry {
    int32_t cls, next;                  // class (-1: none); next entry of the owning lane
    float t;                            // teacher's logit as load_teacher gives it
    Cmp z;                              // student's logit
    float grad;
};

// A teacher's logit: t / Tt, or the bits of an int32, whose list's maximum is taken off in
// integers before anything is rounded.
__device__ __forceinline__ float load_teacher(const DistillArgs &a, int64_t i)
{
    return a.top_type == kI32 ? __int_as_float(load_one<kI32>(a.top_values, i))
                              : load_float(a.top_values, a.top_type, i) * a.inv_top_t;
}
// a maximum to take differences from: 0 where there is none
__device__ __forceinline__ float finite(float m) { return m == -__builtin_inff() ? 0.0f : m; }
// t / Tt, less first / Tt where it is an int32 (first: the largest)
__device__ __forceinline__ float teacher(const DistillArgs &a, float t, int32_t first)
{
    return a.top_type == kI32 ? Elem<kI32>::minus(__float_as_int(t), first) * a.inv_top_t : t;
}
// the given log_norm to go with that
__device__ __forceinline__ float given_norm(const DistillArgs &a, int64_t r, int32_t first)
{
    const float norm = a.top_log_norm[r];
    return a.top_type == kI32 ? norm - (float)first * a.inv_top_t : norm;
}

// GRAD: with the gradient; the loss alone reads the row once and keeps none of it.
template <int TYPE, class L, bool GRAD>
__global__ __launch_bounds__(L::kBlock, GRAD ? L::kWavesPerSimd : 8) void k_distill(DistillArgs a)
{
    typedef Elem<TYPE> E;
    typedef typename E::Cmp Cmp;
    typedef Piece<TYPE, L::VEC> P;
    extern __shared__ uint32_t entries[];                 // [rows of the block][k]
    __shared__ Scratch scratch;
    __shared__ int32_t heads[L::kBlock];                  // first entry of the lane's list
    __shared__ uint32_t marks[L::kBlock];                 // bit j % 32: an entry in piece j
    const int gi = group_of<L::G>();
    const int64_t r = (int64_t)blockIdx.x * L::kGroups + gi;
    if (r >= a.n_rows)
        return;
    Group<L::G> g(threadIdx.x - gi * L::G, &scratch);
    // What the list sums to is worked out by every wave for itself: lists are short, and
    // a reduction over the block costs two of its barriers (4099 x 32003, loss: 67 us with
    // them).
    constexpr int H = L::G < kWave ? L::G : kWave;
    Group<H> h(g.t % H, nullptr);
    Entry<Cmp> *list = reinterpret_cast<Entry<Cmp> *>(entries) + (int64_t)gi * a.k;
    int32_t *head = heads + gi * L::G;
    uint32_t *mark = marks + gi * L::G;
    const char *src = a.logits + r * a.stride;
    char *dst = GRAD ? a.grad + r * a.grad_stride : nullptr;
    const float w = a.row_weight ? a.row_weight[r] : 1.0f;

    Row<TYPE, L::G, L::NV, L::VEC, L::RESIDENT, GRAD> row(src, w == 0.0f ? 0 : a.n, g.t);
    const bool rest = a.top_log_norm != nullptr;
    float Q = 0.0f, S = 0.0f, scale = 0.0f, in_list = 0.0f, outside = 0.0f;
    Cmp from = 0, from_out = 0;
    const Scale c(a.inv_t);
    if (w != 0.0f) {
        head[g.t] = -1;
        mark[g.t] = 0;
        g.barrier();
        for (int e = g.t; e < a.k; e += L::G) {
            const int32_t cls = a.top_indices[r * a.k + e];
            Entry<Cmp> x = {-1, -1, -__builtin_inff(), 0, 0.0f};
            if (cls >= 0 && cls < a.n) {
                x.cls = cls;
                x.t = load_teacher(a, r * a.k + e);
                x.z = load_one<TYPE>(src, cls);
                const int piece = cls / L::VEC, owner = piece % L::G;
                atomicOr(&mark[owner], 1u << (piece / L::G % 32));
                x.next = atomicExch(&head[owner], e);
            }
            list[e] = x;
        }
        g.barrier();
        // the teacher's normalizer: of the list, or given
        float log_norm;
        int32_t first = INT32_MIN;
        if (a.top_type == kI32) {
            for (int e = h.t; e < a.k; e += H)
                if (list[e].cls >= 0)
                    first = max(first, __float_as_int(list[e].t));
            first = h.reduce(first, Max());
        }
        if (rest) {
            log_norm = given_norm(a, r, first);
        } else {
            float tm = -__builtin_inff(), sum = 0.0f;
            if (a.top_type == kI32)
                tm = 0.0f;
            else
                for (int e = h.t; e < a.k; e += H)
                    tm = fmaxf(tm, list[e].t);            // (-inf where there is none)
            tm = finite(h.reduce(tm, Max()));
            for (int e = h.t; e < a.k; e += H)
                if (list[e].cls >= 0)
                    sum += expf(teacher(a, list[e].t, first) - tm);
            sum = h.reduce(sum, Add());
            log_norm = sum == 0.0f ? 0.0f : tm + logf(sum);    // (0: no class, or masked ones)
        }
        Softmax<TYPE> listed;
        for (int e = h.t; e < a.k; e += H)
            if (list[e].cls >= 0) {
                Q += expf(teacher(a, list[e].t, first) - log_norm);
                listed.raise(list[e].z, c.hi);
                listed.s += c.pow(E::minus(list[e].z, listed.from()));
            }
        Q = h.reduce(Q, Add());
        const float q_rest = rest ? fmaxf(0.0f, 1.0f - Q) : 0.0f;

        const uint32_t marked = rest ? mark[g.t] : 0;
        Softmax<TYPE, !L::RESIDENT> sm;
        row.each([&](auto j, int32_t, const P &given) {
            P p = given;
            if (marked >> (j % 32) & 1)
                for (int e = head[g.t]; e >= 0; e = list[e].next)
                    if (list[e].cls / (L::G * L::VEC) == j)
                        p.mask(list[e].cls % L::VEC);
            Cmp z[L::VEC], zm = E::lowest();
#pragma unroll
            for (int u = 0; u < L::VEC; ++u) {
                z[u] = p.get(u);
                zm = Max()(zm, z[u]);
            }
            sm.raise(zm, c.hi);
            const Cmp from = sm.from();
            float part = sm.start();
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                part += c.pow(E::minus(z[u], from));
            sm.add(part);
        });
        // The rest relative to its own maximum, where its mass cannot vanish; the whole
        // row relative to the larger of that and the list's.
        sm = combine(g, sm, c.hi);
        const float s_out = sm.s;
        from_out = sm.from();
        from = from_out;
        float share = 1.0f;                               // e^(from_out - from)
        S = s_out;
        if (rest) {
            listed = combine(h, listed, c.hi);
            const Cmp m = Max()(sm.m, listed.m);
            share = sm.m == m ? 1.0f : c.pow(E::minus(sm.m, m));
            listed.raise(m, c.hi);
            from = listed.from();
            S = s_out * share + listed.s;
        }
        const float log_s = logf(S);
        if (a.loss) {
            float sum = 0.0f;
            for (int e = h.t; e < a.k; e += H)
                if (list[e].cls >= 0) {
                    const float log_q = teacher(a, list[e].t, first) - log_norm, q = expf(log_q);
                    const float log_p = E::minus(list[e].z, from) * a.inv_t - log_s;
                    sum += q == 0.0f ? 0.0f : q * (log_q - log_p);
                }
            sum = h.reduce(sum, Add());
            if (q_rest > 0.0f)
                sum += q_rest * (logf(q_rest) - (E::minus(from_out, from) * a.inv_t +
                                                 logf(s_out) - log_s));
            if (g.t == 0)
                a.loss[r] = w * sum;
        }
        scale = w * a.inv_t;
        if (Q + q_rest == 0.0f)
            scale = 0.0f;                                 // a teacher without classes
        in_list = scale * (Q + q_rest) / S;
        outside = in_list * share;
        if (q_rest > 0.0f)
            outside = s_out == 0.0f && S > 0.0f
                          ? 0.0f : scale * ((Q + q_rest) * share / S - q_rest / s_out);
        if (GRAD) {
            for (int e = g.t; e < a.k; e += L::G)
                if (list[e].cls >= 0)
                    list[e].grad = in_list * c.pow(E::minus(list[e].z, from)) -
                                   scale * expf(teacher(a, list[e].t, first) - log_norm);
            g.barrier();
        }
    } else if (a.loss && g.t == 0) {
        a.loss[r] = 0.0f;
    }
    if constexpr (GRAD) {
        if (scale == 0.0f) {
            const float zero[L::VEC] = {};
            for (int32_t i = 0; i < a.n; i += L::kSpan)
                store_piece<TYPE, L::VEC>(dst, i, g.t * L::VEC, a.n, zero);
            return;
        }
        const uint32_t marked = mark[g.t];
        row.each([&](auto j, int32_t i, const P &p) {
            float v[L::VEC];
            // (the factor's first part: at most 2.5 |z - from| / T 2^-24 of the gradient, of
            // which the rounding of 1 / T is one)
#pragma unroll
            for (int u = 0; u < L::VEC; ++u)
                v[u] = outside * __builtin_amdgcn_exp2f((p.get(u) - from_out) * c.hi);
            if (marked >> (j % 32) & 1)
                for (int e = head[g.t]; e >= 0; e = list[e].next)
                    if (list[e].cls / (L::G * L::VEC) == j) {
#pragma unroll
                        for (int u = 0; u < L::VEC; ++u)
                            if (u == list[e].cls % L::VEC)
                                v[u] = list[e].grad;
                    }
            store_piece<TYPE, L::VEC>(dst, i - g.t * L::VEC, g.t * L::VEC, a.n, v);
        });
    }
}

// Four lanes a row, 16 rows a wave (k <= kLaneEntries): the list's classes leave the tile
// for their entries before it is summed, the exponentials take the logits' places in it,
// then the gradients theirs.  (A lane a row has a quarter of the waves, and their chains
// of LDS accesses take four times as long: 148 us for 262144 rows of 100 float32
// classes with k 10, against 75 here and 112 with a group of 32 lanes and the row in
// registers.  Here the VALU is active in 65 of 100 cycles, the LDS in 19, at 12 waves a
// CU, which the tiles' LDS allows.)
constexpr int32_t kLaneEntries = 32;
// Rows from which on: lanes against groups, float32 with the gradient, k 10, in us:
//   rows        8192      16384      32768      65536     262144
//   10 cl.   7.3, 7.2   7.2, 7.0   7.8, 7.5   9.4, 9.7    27, 30
//   37       7.8, 7.1   7.9, 7.7  8.9, 10.3  12.5, 17.2   34, 56
//   100     10.1, 8.5  10.7, 11.6 13.2, 19.0 18.7, 33.6   58, 113
//   128     10.8, 8.8  11.5, 12.2 14.7, 19.6 25.0, 34.8   88, 130
constexpr int64_t kLaneRows = 16384;
constexpr int kRowLanes = 4;
constexpr int kWaveRows = kWave / kRowLanes;
constexpr int kLaneThreads = 256;

// Rows an odd number of 4 words apart: 16 rows' lanes are in 64 different banks.
__host__ __device__ inline int32_t quad_pitch(int32_t n) { return ((n + 3) / 4 | 1) * 4; }

template <int TYPE>
__global__ __launch_bounds__(kLaneThreads) void k_distill_lanes(DistillArgs a)
{
    typedef Elem<TYPE == kI32 ? kI32 : kF32> E;           // (the tile's elements)
    typedef typename E::Cmp Cmp;
    extern __shared__ uint32_t tiles[];                   // a wave's [16][pitch], and [16][k] of
    const int32_t pitch = quad_pitch(a.n), lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    uint32_t *const tile = tiles + wave * kWaveRows * (pitch + 3 * a.k);
    float *const tops = reinterpret_cast<float *>(tile) + kWaveRows * pitch;   // teacher
    Cmp *const zs = reinterpret_cast<Cmp *>(tops + kWaveRows * a.k);           // student
    int32_t *const classes = reinterpret_cast<int32_t *>(zs + kWaveRows * a.k);
    const int64_t r0 = ((int64_t)blockIdx.x * (kLaneThreads / kWave) + wave) * kWaveRows;
    if (r0 >= a.n_rows)
        return;
    const int32_t rows = (int32_t)min((int64_t)kWaveRows, a.n_rows - r0);
    for (int32_t e = lane; e < rows * a.k; e += kWave) {
        const int32_t cls = a.top_indices[r0 * a.k + e];
        classes[e] = cls >= 0 && cls < a.n ? cls : -1;
        tops[e] = load_teacher(a, r0 * a.k + e);
    }
    load_tile<TYPE>(a.logits + r0 * a.stride, a.stride, rows, a.n, pitch, tile);
    wave_sync();

    Group<kRowLanes> g(lane % kRowLanes, nullptr);
    const int32_t own = lane / kRowLanes;
    if (own < rows) {
        const int64_t r = r0 + own;
        const float w = a.row_weight ? a.row_weight[r] : 1.0f;
        float *z = reinterpret_cast<float *>(tile) + own * pitch;
        const float *top = tops + own * a.k;
        Cmp *scores = reinterpret_cast<Cmp *>(z), *listed = zs + own * a.k;
        const int32_t *cls = classes + own * a.k;
        const Scale c(a.inv_t);
        float scale = 0.0f, loss = 0.0f;
        if (w != 0.0f) {
            // the list leaves the tile; both relative to their own maxima
            Cmp m_list = E::lowest(), m = E::lowest();
            float tm = -__builtin_inff();
            int32_t first = INT32_MIN;
            for (int e = g.t; e < a.k; e += kRowLanes)
                if (cls[e] >= 0) {
                    listed[e] = scores[cls[e]];
                    scores[cls[e]] = E::lowest();
                    m_list = Max()(m_list, listed[e]);
                    tm = fmaxf(tm, top[e]);
                    first = max(first, __float_as_int(top[e]));
                }
            m_list = g.reduce(m_list, Max());
            if (a.top_type == kI32) {
                first = g.reduce(first, Max());
                tm = 0.0f;
            }
            wave_sync();
#pragma unroll 8
            for (int i = g.t; i < a.n; i += kRowLanes)
                m = Max()(m, scores[i]);
            m = g.reduce(m, Max());
            const auto start = [](Cmp v) { return TYPE != kI32 && v == E::lowest() ? 0 : v; };
            const Cmp from_out = start(m);
            const float share = m >= m_list ? 1.0f : c.pow(E::minus(m, m_list));
            m = Max()(m, m_list);
            const Cmp from = start(m);
            float log_norm;
            if (a.top_log_norm) {
                log_norm = given_norm(a, r, first);
            } else {
                tm = finite(g.reduce(tm, Max()));
                float sum = 0.0f;
                for (int e = g.t; e < a.k; e += kRowLanes)
                    sum += cls[e] >= 0 ? expf(teacher(a, top[e], first) - tm) : 0.0f;
                sum = g.reduce(sum, Add());
                log_norm = sum == 0.0f ? 0.0f : tm + logf(sum);    // (0: no class, or masked ones)
            }
            float Q = 0.0f, s_list = 0.0f, s_out = 0.0f;
            for (int e = g.t; e < a.k; e += kRowLanes)
                if (cls[e] >= 0) {
                    Q += expf(teacher(a, top[e], first) - log_norm);
                    s_list += c.pow(E::minus(listed[e], from));
                }
#pragma unroll 8
            for (int i = g.t; i < a.n; i += kRowLanes) {
                const float e = c.pow(E::minus(scores[i], from_out));
                s_out += e;
                z[i] = e;
            }
            Q = g.reduce(Q, Add());
            s_list = g.reduce(s_list, Add());
            s_out = g.reduce(s_out, Add());
            const float S = s_out * share + s_list, log_s = logf(S);
            const float q_rest = a.top_log_norm ? fmaxf(0.0f, 1.0f - Q) : 0.0f;
            if (Q + q_rest != 0.0f)                       // (a teacher without classes)
                scale = w * a.inv_t;
            const float in_list = scale * (Q + q_rest) / S;
            float outside = in_list * share;
            if (q_rest > 0.0f)
                outside = s_out == 0.0f && S > 0.0f
                              ? 0.0f : scale * ((Q + q_rest) * share / S - q_rest / s_out);
            if (a.grad && scale != 0.0f)
#pragma unroll 8
                for (int i = g.t; i < a.n; i += kRowLanes)
                    z[i] *= outside;
            wave_sync();
            for (int e = g.t; e < a.k; e += kRowLanes)
                if (cls[e] >= 0) {
                    const float log_q = teacher(a, top[e], first) - log_norm, q = expf(log_q);
                    const float x = E::minus(listed[e], from) * a.inv_t;
                    loss += q == 0.0f ? 0.0f : q * (log_q - (x - log_s));
                    if (scale != 0.0f)
                        z[cls[e]] = in_list * c.pow(E::minus(listed[e], from)) - scale * q;
                }
            loss = g.reduce(loss, Add());
            if (q_rest > 0.0f)
                loss += q_rest * (logf(q_rest) - (E::minus(from_out, from) * a.inv_t +
                                                  logf(s_out) - log_s));
            loss *= w;
        }
        if (a.loss && g.t == 0)
            a.loss[r] = loss;
        if (a.grad && scale == 0.0f)
            for (int i = g.t; i < a.n; i += kRowLanes)
                z[i] = 0.0f;
    }
    if constexpr (TYPE != kI32) {
        if (!a.grad)
            return;
        wave_sync();
        typedef typename std::conditional<TYPE == kF32, float, typename std::conditional<
            TYPE == kF16, _Float16, __bf16>::type>::type Out;
        const uint32_t inverse = ((1u << 20) + a.n - 1) / a.n, count = (uint32_t)(rows * a.n);
        char *dst = a.grad + r0 * a.grad_stride;
#pragma unroll 4
        for (uint32_t e = lane; e < count; e += kWave) {
            const uint32_t row = e * inverse >> 20, col = e - row * a.n;
            reinterpret_cast<Out *>(dst + row * a.grad_stride)[col] =
                (Out)__uint_as_float(tile[row * pitch + col]);
        }
    }
}

}  // namespace

hipError_t launch_distill(const void *logits, int32_t type, int64_t n_rows, int32_t n,
                          int64_t row_stride, float inv_t, const void *top_values,
                          int32_t top_type, const int32_t *top_indices, int32_t k,
                          const float *top_log_norm, float inv_top_t, const float *row_weight,
                          float *loss, void *grad, int64_t grad_stride, hipStream_t stream)
{
    return with_type(type, [&](auto ty) {
        constexpr int TYPE = decltype(ty)::value;
        const DistillArgs a = {static_cast<const char *>(logits),
                               row_stride * Elem<TYPE>::kBytes, n_rows, n, k, top_type, inv_t,
                               inv_top_t, static_cast<const char *>(top_values), top_indices,
                               top_log_norm, row_weight, loss, static_cast<char *>(grad),
                               grad_stride * Elem<TYPE>::kBytes};
        if (n <= kLaneClasses && k <= kLaneEntries && n_rows >= kLaneRows) {
            constexpr int kRows = kLaneThreads / kRowLanes;
            const size_t words = (size_t)kRows * (quad_pitch(n) + 3 * k);
            return in_launches(a, kLaneThreads, kRows,
                               [&](const DistillArgs &part, uint32_t blocks) {
                k_distill_lanes<TYPE><<<blocks, kLaneThreads, words * 4, stream>>>(part);
            });
        }
        return with_layout<TYPE>(n, k, [&](auto layout) {
            typedef decltype(layout) L;
            const size_t lds = (size_t)L::kGroups * k * sizeof(Entry<float>);
            return in_launches(a, L::kBlock, L::kGroups,
                               [&](const DistillArgs &part, uint32_t blocks) {
                if constexpr (TYPE != kI32)
                    if (grad) {
                        k_distill<TYPE, L, true><<<blocks, L::kBlock, lds, stream>>>(part);
                        return;
                    }
                k_distill<TYPE, L, false><<<blocks, L::kBlock, lds, stream>>>(part);
            });
        });
    });
}

}  // namespace bl
