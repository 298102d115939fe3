// 8-bit levels with a scale for each row, and the product of two such matrices (include/dqn_mi355.h: q8_quantize_rows, q8_linear).
#include "quant.h"

#include "gemm_mfma.h"

namespace dqn {

// ---- rows to levels -------------------------------------------------------------------------------------------------
//
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

// What a level stands for.  127 times a scale that was rounded up can lie beyond the largest fp32 number: the row's own maximum does not.
__device__ inline float level_value(int q, float s)
{
    const float v = static_cast<float>(q) * s;
    return v > 0x1.fffffep127f ? 0x1.fffffep127f : v < -0x1.fffffep127f ? -0x1.fffffep127f : v;   // (a NaN stays)
}

template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* x, int64_t ldx, int64_t cols, int8_t* q, int64_t ldq, float* scale, T* values, int64_t ldv)
{
    __shared__ uint32_t part[4];
    const int64_t row = blockIdx.x;
    x += row * ldx;
    uint32_t top = 0;   // bits of |x|: they order as the values do, infinities and NaN above all others
    for (int64_t c = threadIdx.x; c < cols; c += 256) top = max(top, __float_as_uint(fabsf(static_cast<float>(x[c]))));
    for (int d = 32; d; d >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), d)));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(part[0], part[1]), max(part[2], part[3]));
    const bool finite = top < 0x7F800000u;
    const float a = finite ? __uint_as_float(top) : 0.f, s = finite ? row_scale(a) : __uint_as_float(0x7FC00000u);
    const Levels l = make_levels(a);
    for (int64_t c = threadIdx.x; c < cols; c += 256) {
        const int v = finite ? level_of(l, static_cast<float>(x[c])) : 0;
        if (q) q[row * ldq + c] = static_cast<int8_t>(v);
        if (values) values[row * ldv + c] = static_cast<T>(level_value(v, s));
    }
    if (threadIdx.x == 0) scale[row] = s;
}

template <typename T>
static void launch_quantize(const void* x, int64_t ldx, int64_t rows, int64_t cols, int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv, hipStream_t st)
{
    hipLaunchKernelGGL(quantize_rows_kernel<T>, dim3(static_cast<unsigned>(rows)), dim3(256), 0, st, static_cast<const T*>(x), ldx, cols, q, ldq, scale, static_cast<T*>(values), ldv);
}

int enqueue_quantize_rows(const void* x, int32_t type, int64_t ldx, int64_t rows, int64_t cols, int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv,
                          hipStream_t st)
{
    auto launch = type == DQN_TYPE_FP32 ? launch_quantize<float> : type == DQN_TYPE_BF16 ? launch_quantize<bf16_t> : launch_quantize<_Float16>;
    launch(x, ldx, rows, cols, q, ldq, scale, values, ldv, st);
    DQN_LAUNCH_CHECK();
    return DQN_OK;
}

// ---- y = act(sx sw (x w^T) + b) ----------------------------------------------------------------------------------------

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct Q8Args {
    const int8_t* x; const int8_t* w;
    const float* sx; const float* sw; const float* bias;   // bias may be null
    void* y;
    int64_t ldx, ldw, ldy;
    int M, N, K, relu;
};

// The sum is exact in 32-bit integers; scales and bias are applied in fp64 (their product neither overflows nor underflows there, and
// only the result is rounded) and the result is rounded once to y's type.
template <typename T> __device__ inline T q8_result(int32_t acc, float sx, float sw, float b, bool relu)
{
    const float v = static_cast<float>(static_cast<double>(acc) * (static_cast<double>(sx) * static_cast<double>(sw)) + static_cast<double>(b));
    return static_cast<T>(relu && v < 0.f ? 0.f : v);   // (a NaN stays)
}

// 16 levels of a row from column k on; zeros from column K on and for rows that there are none of.
__device__ inline i32x4 q8_load(const int8_t* row, int k, int K, bool in)
{
    i32x4 v = {0, 0, 0, 0};
    if (!in || k >= K) return v;
    if (k + 16 <= K) {
        __builtin_memcpy(&v, row + k, 16);
        return v;
    }
    uint8_t b[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) b[i] = k + i < K ? static_cast<uint8_t>(row[k + i]) : 0;
    __builtin_memcpy(&v, b, 16);
    return v;
}

template <typename T>
__global__ __launch_bounds__(256) void q8_linear_kernel(Q8Args a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int m0 = static_cast<int>(blockIdx.y) * 16, n0 = (static_cast<int>(blockIdx.x) * 4 + wave) * 16, r = lane & 15, kq = 16 * (lane >> 4);
    const bool in_m = m0 + r < a.M, in_n = n0 + r < a.N;
    const int8_t* x = a.x + static_cast<int64_t>(in_m ? m0 + r : 0) * a.ldx;
    const int8_t* w = a.w + static_cast<int64_t>(in_n ? n0 + r : 0) * a.ldw;
    i32x4 acc = {0, 0, 0, 0};
    for (int k = 0; k < a.K; k += 64) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(q8_load(x, k + kq, a.K, in_m), q8_load(w, k + kq, a.K, in_n), acc, 0, 0, 0);
    if (!in_n) return;
    const float sw = a.sw[n0 + r], b = a.bias ? a.bias[n0 + r] : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + 4 * (lane >> 4) + i;
        if (m < a.M) static_cast<T*>(a.y)[m * a.ldy + n0 + r] = q8_result<T>(acc[i], a.sx[m], sw, b, a.relu);
    }
}

int enqueue_q8_linear(const int8_t* x, int64_t ldx, const float* sx, const int8_t* w, int64_t ldw, const float* sw, const float* bias, bool relu, int64_t M,
                      int64_t N, int64_t K, void* y, int32_t type, int64_t ldy, hipStream_t st)
{
    Q8Args a{x, w, sx, sw, bias, y, ldx, ldw, ldy, static_cast<int>(M), static_cast<int>(N), static_cast<int>(K), relu};
    auto kern = type == DQN_TYPE_FP32 ? q8_linear_kernel<float> : type == DQN_TYPE_BF16 ? q8_linear_kernel<bf16_t> : q8_linear_kernel<_Float16>;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>((N + 63) / 64), static_cast<unsigned>((M + 15) / 16)), dim3(256), 0, st, a);
    DQN_LAUNCH_CHECK();
    return DQN_OK;
}

}  // namespace dqn

using namespace dqn;

extern "C" {

int q8_quantize_rows(const void* x, int32_t type, int64_t ldx, int64_t rows, int64_t cols, int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv,
                     void* stream)
{
    const char* who = "q8_quantize_rows";
    if (int rc = check_type(who, type)) return rc;
    if (rows < 0 || rows > Q8_QUANTIZE_MAX_ROWS || cols < 0 || cols > INT32_MAX) return fail(DQN_EINVAL, "%s: rows = %lld, cols = %lld", who, (long long)rows, (long long)cols);
    if (rows == 0) return DQN_OK;
    if (!scale || (cols && (!x || (!q && !values)))) return fail(DQN_EINVAL, "%s: null pointer", who);
    const uintptr_t e = type == DQN_TYPE_FP32 ? 4 : 2;
    if (!aligned_to(x, e) || !aligned_to(values, e) || !aligned_to(scale, 4)) return fail(DQN_EINVAL, "%s: a pointer is not aligned to its elements", who);
    if (ldx < cols || (q && ldq < cols) || (values && ldv < cols)) return fail(DQN_EINVAL, "%s: a row pitch is shorter than a row", who);
    if (int rc = check_stream_device(who, stream)) return rc;
    return enqueue_quantize_rows(x, type, ldx, rows, cols, q, ldq, scale, values, ldv, static_cast<hipStream_t>(stream));
}

int q8_linear(const int8_t* x, int64_t ldx, const float* sx, const int8_t* w, int64_t ldw, const float* sw, const float* bias, int32_t relu, int64_t M, int64_t N,
              int64_t K, void* y, int32_t type, int64_t ldy, void* stream)
{
    const char* who = "q8_linear";
    if (int rc = check_type(who, type)) return rc;
    if (M < 0 || M > Q8_LINEAR_MAX_ROWS || N < 0 || N > Q8_LINEAR_MAX_ROWS) return fail(DQN_EINVAL, "%s: M = %lld, N = %lld outside 0..%d", who, (long long)M, (long long)N, Q8_LINEAR_MAX_ROWS);
    if (K < 0 || K > Q8_LINEAR_MAX_K) return fail(DQN_EINVAL, "%s: K = %lld outside 0..%d", who, (long long)K, Q8_LINEAR_MAX_K);
    if (M == 0 || N == 0) return DQN_OK;
    if (!sx || !sw || !y || (K && (!x || !w))) return fail(DQN_EINVAL, "%s: null pointer", who);
    if (!aligned_to(y, type == DQN_TYPE_FP32 ? 4 : 2) || !aligned_to(sx, 4) || !aligned_to(sw, 4) || !aligned_to(bias, 4))
        return fail(DQN_EINVAL, "%s: a pointer is not aligned to its elements", who);
    if (ldx < K || ldw < K || ldy < N) return fail(DQN_EINVAL, "%s: a row pitch is shorter than a row", who);
    if (int rc = check_stream_device(who, stream)) return rc;
    return enqueue_q8_linear(x, ldx, sx, w, ldw, sw, bias, relu != 0, M, N, K, y, type, ldy, static_cast<hipStream_t>(stream));
}

}  // extern "C"
