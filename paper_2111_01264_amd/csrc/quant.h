// Row quantisation to 8-bit levels and the product of such levels: what net.hip and the C entries of quant.hip share.
#pragma once
#include "common.h"

namespace dqn {

// Enqueue only; arguments have been checked.
int enqueue_quantize_rows(const void* x, int32_t type, int64_t ldx, int64_t rows, int64_t cols, int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv,
                          hipStream_t st);
int enqueue_q8_linear(const int8_t* x, int64_t ldx, const float* sx, const int8_t* w, int64_t ldw, const float* sw, const float* bias, bool relu, int64_t M,
                      int64_t N, int64_t K, void* y, int32_t type, int64_t ldy, hipStream_t st);

// scale = fl(a / 127), level = rint(127 x / a) with a = max |x| of the row.  The level is rint of the EXACT quotient: the fp32 quotient
// is off by less than 2^-15 of a level, so only a value that close to the border between two levels is decided again, in fp64, where
// 127 x - level a has no rounding.
__device__ inline float row_scale(float a) { return static_cast<float>(static_cast<double>(a) / 127.0); }

struct Levels {
    float a, inv;   // the row's largest magnitude and 127 / a, both times `up`
    float up;       // 2^64 where a is so small that 127 / a would overflow, else 1
};
__device__ inline Levels make_levels(float a)
{
    Levels l;
    l.up = a < 0x1p-100f ? 0x1p64f : 1.f;
    l.a = a * l.up;
    l.inv = a > 0.f ? 127.f / l.a : 0.f;
    return l;
}
__device__ inline int level_of(const Levels& l, float x)
{
    x *= l.up;
    const float f = x * l.inv;
    float q = rintf(f);
    if (fabsf(fabsf(f - q) - 0.5f) < 0x1p-13f) {
        const double a = l.a, r = 127.0 * x - static_cast<double>(q) * a;   // exact
        const bool odd = static_cast<int>(q) & 1;
        if (2.0 * r > a || (2.0 * r == a && odd)) q += 1.f;
        else if (2.0 * r < -a || (2.0 * r == -a && odd)) q -= 1.f;
    }
    return static_cast<int>(q);
}

template <typename T> __device__ inline uint32_t magnitude(T v) { return __float_as_uint(fabsf(static_cast<float>(v))); }   // they order as the values do, infinities and NaN above all others

// The sum is exact in 32-bit integers; scales and bias are applied in fp64 (their product neither overflows nor underflows there, and
// only the result is rounded) and the result is rounded to fp32 and to y's type.  floor: 0 with a ReLU, else -infinity; a NaN stays.
template <typename T> __device__ inline T q8_result(int32_t acc, float sx, float sw, float b, float floor)
{
    const float v = static_cast<float>(static_cast<double>(acc) * (static_cast<double>(sx) * static_cast<double>(sw)) + static_cast<double>(b));
    return static_cast<T>(v < floor ? floor : v);
}

}  // namespace dqn
