// Dropout whose mask is a function of (seed, offset, row, column): computed where it is
// needed, in the forward pass and again in the backward pass, and never stored.
//
// Eight elements of a row share a counter (column / 8, row, offset): Philox 4x32 with ten
// rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011) turns it into four words, eight numbers of 16 bits.  An element stays where its
// number is at least round(p 2^16).  Sixteen bits a number halve the generator's work a
// byte; what they cost is that p is one of 2^16 + 1 values, and the factor of the elements
// that stay is the exact reciprocal of that value's complement, so the mean is unbiased.
//
// Memory bounds it: a copy's bytes.  16384 x 8192 in bf16 takes 99 us where torch's copy of
// it takes 100, 2^18 x 100 counts 49 us where their copy as float takes 67 (42 where they are in
// the caches); with one round for ten 88 and 49 us, so the products mostly hide behind the
// loads.  In odd rows, 16381 x 8191, they show: 103 to 145 us, with one round 95 to 101.  Lanes of
// eight elements load and store 16 or 32 bytes.
#include "logit_rows.h"

namespace bl {
namespace {

using namespace rows;

constexpr int kBlock = 256;
constexpr int kEight = 8;

struct DropoutArgs {
    const char *x;
    int64_t stride;                     // bytes from row to row
    int64_t n_rows;
    int32_t n, eights;                  // columns, and counters of a row
    char *out;
    int64_t out_stride;
    uint32_t border;                    // numbers below are dropped; 65536: all
    float factor;
    uint64_t seed, offset;
    const uint64_t *offset_at;          // added to offset where not NULL
};

// The four words of a counter: ten rounds of two 32 x 32 bit products.
__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
        c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0;
        c[1] = (uint32_t)b;
        c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1;
        c[3] = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// to_bits: the result's bits, rounded once from 32 (to the nearest, ties to even).
template <int TYPE>
__device__ __forceinline__ uint32_t to_bits(float v)
{
    if constexpr (TYPE == kF16) {
        const _Float16 h = (_Float16)v;
        uint16_t b;
        __builtin_memcpy(&b, &h, 2);
        return b;
    } else if constexpr (TYPE == kBf16) {
        const __bf16 h = (__bf16)v;
        uint16_t b;
        __builtin_memcpy(&b, &h, 2);
        return b;
    } else {
        return __float_as_uint(v);
    }
}

// The first of N words moved down by `by` elements of `bytes` bytes, a bit of it at a time.
template <int N>
__device__ __forceinline__ void move_down(uint32_t (&w)[N], int by, int bytes)
{
    const int words = by * bytes / 4;
#pragma unroll
    for (int step = 1; step < N; step *= 2)
#pragma unroll
        for (int k = 0; k < N; ++k)
            w[k] = words & step ? (k + step < N ? w[k + step] : 0u) : w[k];
    if (bytes == 2 && (by & 1)) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            w[k] = w[k] >> 16 | (k + 1 < N ? w[k + 1] << 16 : 0u);
    }
}

// The last eight elements of a row, moved down to those from i on: one load, where a loop
// over them, each waiting for the one before, took 133 us for 16381 x 8191 in bf16, not 107.
// (In place, a neighbour may have stored some of them already: those are moved out.)
template <int TYPE>
__device__ __forceinline__ void load_row(Piece<TYPE, kEight> &p, const char *row, int32_t i,
                                         int32_t n)
{
    constexpr int B = Elem<TYPE>::kBytes;
    if (n < kEight) {                                     // (in the whole wave)
        p.load(row, 0, i, n);
        return;
    }
    const int32_t at = min(i, n - kEight);
    __builtin_memcpy(p.w, row + (int64_t)at * B, sizeof p.w);
    if (at < i)
        move_down(p.w, i - at, B);
}

// The first `count` (below eight) of eight elements stored, four, two and one at a time.
template <int N>
__device__ __forceinline__ void store_end(char *dst, uint32_t (&w)[N], int count)
{
    constexpr int B = N / 2;                              // bytes of an element: 2, 4
#pragma unroll
    for (int some = 4; some; some /= 2)
        if (count & some) {
            __builtin_memcpy(dst, w, (size_t)some * B);
            dst += some * B;
            move_down(w, some, B);
        }
}

template <int TYPE>
__global__ __launch_bounds__(kBlock) void k_dropout(DropoutArgs a, uint64_t tasks)
{
    constexpr int kBytes = Elem<TYPE>::kBytes;
    uint64_t offset = a.offset;
    if (a.offset_at)
        offset += *a.offset_at;
    // a block's tasks (eight columns each) are consecutive: one 64-bit division a
    // block and a 32-bit one a lane find their rows
    for (uint64_t first = (uint64_t)blockIdx.x * kBlock; first < tasks;
         first += (uint64_t)gridDim.x * kBlock) {
        const uint64_t row0 = first / (uint32_t)a.eights;
        const uint32_t at = (uint32_t)(first - row0 * (uint32_t)a.eights) + threadIdx.x;
        if (first + threadIdx.x >= tasks)
            return;
        const uint32_t down = at / (uint32_t)a.eights, eight = at - down * (uint32_t)a.eights;
        const uint64_t row = row0 + down;
        const int32_t i = (int32_t)(eight * kEight);
        const char *src = a.x + row * a.stride;
        char *dst = a.out + row * a.out_stride + (int64_t)i * kBytes;
        Piece<TYPE, kEight> p;
        load_row(p, src, i, a.n);
        uint32_t c[4] = {eight, (uint32_t)row, (uint32_t)offset, (uint32_t)(offset >> 32)};
        philox(c, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
        uint32_t w[kEight];
#pragma unroll
        for (int u = 0; u < kEight; ++u) {
            const uint32_t number = u & 1 ? c[u / 2] >> 16 : c[u / 2] & 0xFFFFu;
            const float v = Elem<TYPE>::to_float(p.get(u)) * a.factor;
            w[u] = to_bits<TYPE>(number >= a.border ? v : 0.0f);
        }
        if constexpr (kBytes == 2) {
            uint32_t packed[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                packed[u] = w[2 * u] | w[2 * u + 1] << 16;
            if (i + kEight <= a.n)
                __builtin_memcpy(dst, packed, sizeof packed);
            else
                store_end(dst, packed, a.n - i);
        } else {
            if (i + kEight <= a.n)
                __builtin_memcpy(dst, w, sizeof w);
            else
                store_end(dst, w, a.n - i);
        }
    }
}

}  // namespace

hipError_t launch_dropout(const void *x, int32_t type, int64_t n_rows, int32_t n,
                          int64_t row_stride, uint32_t border, uint64_t seed, uint64_t offset,
                          const uint64_t *offset_at, void *out, int64_t out_stride,
                          hipStream_t stream)
{
    const int32_t eights = (n + kEight - 1) / kEight;
    const uint64_t tasks = (uint64_t)n_rows * (uint32_t)eights;
    const float factor = border < 65536 ? (float)(65536.0 / (65536 - border)) : 0.0f;
    const uint64_t blocks = (tasks + kBlock - 1) / kBlock;
    const uint32_t grid = (uint32_t)(blocks < (1u << 20) ? blocks : (1u << 20));
    return with_type(type, [&](auto T) {
        constexpr int TYPE = decltype(T)::value;
        const DropoutArgs a = {static_cast<const char *>(x), row_stride * Elem<TYPE>::kBytes,
                               n_rows, n, eights, static_cast<char *>(out),
                               out_stride * Elem<TYPE>::kBytes, border, factor, seed, offset,
                               offset_at};
        hipLaunchKernelGGL(k_dropout<TYPE>, dim3(grid), dim3(kBlock), 0, stream, a, tasks);
        return hipGetLastError();
    });
}

}  // namespace bl
