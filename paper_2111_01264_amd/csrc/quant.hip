// 8-bit levels with a scale for each row, and the product of two such matrices (include/dqn_mi355.h: q8_quantize_rows, q8_linear).
#include <type_traits>

#include "quant.h"

#include "gemm_mfma.h"

namespace dqn {

// ---- rows to levels -------------------------------------------------------------------------------------------------
//
// What a level stands for.  127 times a scale that was rounded up can lie beyond the largest fp32 number: the row's own maximum does not.
__device__ inline float level_value(int q, float s)
{
    const float v = static_cast<float>(q) * s;
    return v > 0x1.fffffep127f ? 0x1.fffffep127f : v < -0x1.fffffep127f ? -0x1.fffffep127f : v;   // (a NaN stays)
}

template <typename T> struct Vec16 {   // 16 bytes of a row, at any alignment that its elements have
    static constexpr int E = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    typedef int8_t levels __attribute__((ext_vector_type(E), aligned(1)));
};

struct QuantArgs { const void* x; int8_t* q; float* scale; void* values; int64_t ldx, ldq, ldv; int64_t rows; int cols; };

// Memory bounds it, so a row is read once: TPR threads hold it, R vectors of 16 bytes each, find its largest magnitude and write the levels.
// A row beyond TPR * R vectors (R = 0) is read twice, the second time from cache.  8192x8192 bf16 with values: 64 us, 5.3 TB/s, as fast as a copy (read twice, in single
// elements: 154 us); 1001x5003 fp32 in a wider matrix: 10.4 us, 4.3 TB/s.
template <typename T, int TPR, int R>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void quantize_rows_kernel(QuantArgs a)
{
    typedef typename Vec16<T>::type vec;
    typedef typename Vec16<T>::levels vec_q;
    constexpr int E = Vec16<T>::E, RPB = TPR < 256 ? 256 / TPR : 1;   // rows per workgroup
    const int64_t row = blockIdx.x * static_cast<int64_t>(RPB) + threadIdx.x / TPR;
    if (TPR < 256 && row >= a.rows) return;   // (a wavefront's row, and no barrier below)
    const int t = threadIdx.x % TPR, cols = a.cols, vecs = (cols + E - 1) / E;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    auto load = [&](int v) {   // zeros behind the end
        vec w;
        if ((v + 1) * E <= cols) w = *reinterpret_cast<const vec*>(x + v * E);
        else {
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = v * E + e < cols ? x[v * E + e] : static_cast<T>(0.f);
        }
        return w;
    };
    uint32_t top = 0;
    vec held[R ? R : 1];
    if constexpr (R > 0) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i * TPR + t < vecs) held[i] = load(i * TPR + t);
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i * TPR + t < vecs) {
#pragma unroll
                for (int e = 0; e < E; ++e) top = max(top, magnitude(held[i][e]));
            }
    } else {
        for (int v = t; v < vecs; v += TPR) {
            const vec w = load(v);
#pragma unroll
            for (int e = 0; e < E; ++e) top = max(top, magnitude(w[e]));
        }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), d)));
    if constexpr (TPR > 64) {
        __shared__ uint32_t part[TPR / 64];
        if ((t & 63) == 0) part[t >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) top = max(top, part[i]);
    }
    const bool finite = top < 0x7F800000u;
    const float m = finite ? __uint_as_float(top) : 0.f, s = finite ? row_scale(m) : __uint_as_float(0x7FC00000u);
    const Levels l = make_levels(m);
    int8_t* q = a.q ? a.q + row * a.ldq : nullptr;
    T* values = a.values ? static_cast<T*>(a.values) + row * a.ldv : nullptr;
    auto write = [&](int v, const vec& w) {
        vec_q lev;
        vec val;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int n = finite ? level_of(l, static_cast<float>(w[e])) : 0;
            lev[e] = static_cast<int8_t>(n);
            val[e] = static_cast<T>(level_value(n, s));
        }
        if ((v + 1) * E <= cols) {
            if (q) *reinterpret_cast<vec_q*>(q + v * E) = lev;
            if (values) *reinterpret_cast<vec*>(values + v * E) = val;
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (v * E + e < cols) {
                    if (q) q[v * E + e] = lev[e];
                    if (values) values[v * E + e] = val[e];
                }
        }
    };
    if constexpr (R > 0) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i * TPR + t < vecs) write(i * TPR + t, held[i]);
    } else {
        for (int v = t; v < vecs; v += TPR) write(v, load(v));
    }
    if (t == 0) a.scale[row] = s;
}

template <typename T> static void launch_quantize(const QuantArgs& a, hipStream_t st)
{
    const int vecs = (a.cols + Vec16<T>::E - 1) / Vec16<T>::E;
    const auto go = [&](auto kern, int tpr) {
        const int rpb = tpr < 256 ? 256 / tpr : 1;
        hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>((a.rows + rpb - 1) / rpb)), dim3(tpr < 256 ? 256 : tpr), 0, st, a);
    };
    // The smallest workgroup that holds a row in few vectors, but all of a compute unit's threads for a row where rows are few.  Levels alone, in us, 64 / 256 threads: 8192 rows of 1024 bf16
    // 9.8 / 13.0; 256 with four / eight vectors: 8192 rows of 8192 43.7 / 44.0; 256 / 1024: 32 rows of 2048 3.4 / 3.7, of 3136 4.3 / 3.8, of 8192 6.0 / 4.7, of 16384 12.7 / 6.9; 512 rows of
    // 3136 5.4 / 5.5, of 8192 8.4 / 7.1, of 16384 14.6 / 11.2; 1024 of 8192 10.5 / 11.4, of 16384 20 / 18; 2048 of 8192 17.6 / 19.5; 8192 of 8192 44 / 63.  Read once / twice: 1024 rows of
    // 65536 54 / 58, fp32 of 32768 35 / 44.
    if (vecs <= 64 * 2) go(quantize_rows_kernel<T, 64, 2>, 64);
    else if (a.rows <= 512 && vecs > 384 && vecs <= 1024 * 8) go(quantize_rows_kernel<T, 1024, 8>, 1024);
    else if (vecs <= 256 * 4) go(quantize_rows_kernel<T, 256, 4>, 256);
    else if (vecs <= 256 * 8) go(quantize_rows_kernel<T, 256, 8>, 256);
    else if (vecs <= 1024 * 8) go(quantize_rows_kernel<T, 1024, 8>, 1024);
    else go(quantize_rows_kernel<T, 1024, 0>, 1024);
}

int enqueue_quantize_rows(const void* x, int32_t type, int64_t ldx, int64_t rows, int64_t cols, int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv,
                          hipStream_t st)
{
    const QuantArgs a{x, q, scale, values, ldx, ldq, ldv, rows, static_cast<int>(cols)};
    type == DQN_TYPE_FP32 ? launch_quantize<float>(a, st) : type == DQN_TYPE_BF16 ? launch_quantize<bf16_t>(a, st) : launch_quantize<_Float16>(a, st);
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

// 16 levels of a row from column k on; zeros from column K on.
__device__ inline i32x4 q8_load(const int8_t* row, int k, int K)
{
    i32x4 v = {0, 0, 0, 0};
    if (k >= K) return v;
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

// The 32x32 matrix instruction on 8-bit operands (the 16x16 one alike): lane l feeds row l % 32 with 16 levels of k, the lanes below 32 and the others
// with different ones, and receives column l % 32 with rows 8 (v / 4) + 4 (l / 32) + v % 4, v = 0 .. 15.  Which 16 of a tile's k a lane
// feeds is free as long as both operands agree.  w is the first operand everywhere, so that a lane holds one row m of y and four columns n in a row.
typedef int i32x16 __attribute__((ext_vector_type(16)));
__device__ inline i32x16 q8_mma(const i32x4& w, const i32x4& x, const i32x16& acc) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(w, x, acc, 0, 0, 0); }
__device__ inline i32x4 q8_mma(const i32x4& w, const i32x4& x, const i32x4& acc) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc, 0, 0, 0); }

// Four columns n .. n + 3 of y as they leave the matrix instructions: their scales and biases once, then the rows m that this lane has of them.
struct Q8Columns {
    float sw[4], b[4], floor;
    int n, left;   // columns of them that there are
};
__device__ inline Q8Columns q8_columns(const Q8Args& a, int n)
{
    Q8Columns c;
    c.n = n; c.left = a.N - n;
    c.floor = a.relu ? 0.f : -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = min(n + i, a.N - 1);
        c.sw[i] = a.sw[at];
        c.b[i] = a.bias ? a.bias[at] : 0.f;
    }
    return c;
}
template <typename T> __device__ inline void q8_store(const Q8Args& a, const Q8Columns& c, int m, float sx, int32_t v0, int32_t v1, int32_t v2, int32_t v3)
{
    typedef T T4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const int32_t v[4] = {v0, v1, v2, v3};
    T4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = q8_result<T>(v[i], sx, c.sw[i], c.b[i], c.floor);
    if (m >= a.M) return;
    T* y = static_cast<T*>(a.y) + m * a.ldy + c.n;
    if (c.left >= 4) *reinterpret_cast<T4*>(y) = out;
    else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < c.left) y[i] = out[i];
    }
}

// ---- few rows: the weights are streamed once, from memory straight into the matrix instructions ---------------------------------
//
// A workgroup owns BN rows of w and BN rows of x; its wavefronts take every WAVES-th stretch of k
// and meet in LDS at the end.  No staging: a row of w is used by one wavefront only, and the rows of x come from cache.  Memory's latency bounds it, so a
// stretch's U loads of either side are requested while the one before is multiplied, and what is left behind the last stretch before anything else.
// 1x16384x4096: 13.0 us, 5.2 TB/s; 512x512x3136: 7.9 us (each stretch's loads behind the last stretch's products: 9.4); 8x512x3136: 5.6 us, as long as any call.
template <typename T, int BN, int U, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void q8_stream_kernel(Q8Args a)
{
    typedef typename std::conditional<BN == 16, i32x4, i32x16>::type acc_t;
    constexpr int KI = BN == 16 ? 64 : 32, V = BN == 16 ? 4 : 16;   // k of one instruction, results per lane
    static_assert(U <= WAVES, "less than a stretch is left: one instruction per wavefront at most");
    __shared__ int32_t part[(WAVES - 1) * V * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = static_cast<int>(blockIdx.x) * BN, m0 = static_cast<int>(blockIdx.y) * BN, r = lane % BN, kq = 16 * (lane / BN);
    const int8_t* w = a.w + static_cast<int64_t>(min(n0 + r, a.N - 1)) * a.ldw + kq;   // (rows past the end repeat the last one: their results are not stored)
    const int8_t* x = a.x + static_cast<int64_t>(min(m0 + r, a.M - 1)) * a.ldx + kq;
    acc_t acc;
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = 0;
    const int K = a.K, whole = K / (KI * U), rest = whole * (KI * U) + wave * KI;
    const i32x4 w_rest = q8_load(w, rest, K - kq), x_rest = q8_load(x, rest, K - kq);
    i32x4 wf[2][U], xf[2][U];
    auto load = [&](int s, int to) {
#pragma unroll
        for (int u = 0; u < U; ++u) __builtin_memcpy(&wf[to][u], w + s * (KI * U) + u * KI, 16);
#pragma unroll
        for (int u = 0; u < U; ++u) __builtin_memcpy(&xf[to][u], x + s * (KI * U) + u * KI, 16);
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int u = 0; u < U; ++u) acc = q8_mma(wf[from][u], xf[from][u], acc);
    };
    if (wave < whole) load(wave, 0);
    for (int s = wave; s < whole; s += 2 * WAVES) {
        if (s + WAVES < whole) load(s + WAVES, 1);
        multiply(0);
        if (s + WAVES >= whole) break;
        if (s + 2 * WAVES < whole) load(s + 2 * WAVES, 0);
        multiply(1);
    }
    acc = q8_mma(w_rest, x_rest, acc);
    if (wave > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) part[((wave - 1) * V + v) * 64 + lane] = acc[v];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int q = 0; q < WAVES - 1; ++q)
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] += part[(q * V + v) * 64 + lane];
    const int m = m0 + r;
    const float sx = a.sx[min(m, a.M - 1)];
#pragma unroll
    for (int g = 0; g < V / 4; ++g) {
        const Q8Columns c = q8_columns(a, n0 + (BN == 16 ? 4 * (lane / BN) : 8 * g + 4 * (lane / BN)));
        q8_store<T>(a, c, m, sx, acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]);
    }
}

// ---- many rows: tiles staged through LDS -----------------------------------------------------------------------------------
//
// THREADS threads own a TILE x TILE piece of y, each wavefront a part of it.  k advances in steps of 64: a stage holds 64 levels of TILE rows of x and
// of w, four of them are in LDS, and the loads go straight from memory into LDS, those of two steps (a cache line of each row) together, as soon as two stages are
// free.  A wavefront reads the operands of the next half step while it multiplies those of this one; there is one barrier per step, in the middle: behind it the
// stage that everybody has read is free, and the next one is complete.  Rows that do not start on 16-byte borders (not ALIGNED) come through registers, a step ahead.
//
// 8192^3: 550 to 615 us, 1.8 to 2.0 PTOP/s; what bounds it is power: the matrix instructions need 524 k cycles of each SIMD (218 us at 2.4 GHz), 54 % of the 967 k that a launch takes at a clock
// of 1.65 GHz; levels that are all zero take 420 us (profiles/actor_operators_counters.txt).  One wavefront per SIMD with parts of 128 x 128 takes as long as two of 128 x 64.
// 1111x2051x2003: 20 us, packed 28.
//
// A row's four 16-byte chunks are stored at the places c ^ swizzle(row), so that the 32 rows that one read takes the same chunk of do
// not meet in the same banks.
constexpr int kStep = 64, kStages = 4;
__device__ inline int q8_swizzle(int row) { return (((row >> 1) ^ (row >> 3)) & 1) | ((row >> 1) & 2); }

// 16 bytes per lane from base + offset (which differs per lane) into LDS at the wavefront's `lds` + 16 * lane.  Nothing but q8_wait waits for them.
__device__ inline void q8_to_lds(const int8_t* base, uint32_t offset, uint32_t lds)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base + offset), (__attribute__((address_space(3))) void*)static_cast<uintptr_t>(lds), 16, 0, 0);
}
template <int LEFT> __device__ inline void q8_wait() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LEFT) : "memory"); }

template <typename T, int TILE, int THREADS, bool ALIGNED>
__global__ __launch_bounds__(THREADS, TILE == 256 ? THREADS / 256 : TILE == 128 ? 2 : 4) void q8_tile_kernel(Q8Args a, int tiles_m, int tiles_n)
{
    constexpr int WN = THREADS / 128, FX = TILE / 64, FW = TILE / WN / 32;   // the wavefronts' parts: WN along n, two along m; 32-row operand tiles of each
    constexpr int kHalf = TILE * kStep, kStage = 2 * kHalf;        // bytes: w's rows, then x's
    constexpr int L = kStage / 16 / THREADS;                          // 16-byte loads per thread and step
    extern __shared__ __attribute__((aligned(128))) int8_t q8_smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // Workgroups go to the eight XCDs in turn, each with an L2 of its own: an XCD takes a contiguous eighth of the tiles, in strips of eight
    // tile rows, so that the tiles that are worked on together share rows of x and w.
    int tm, tn;
    {
        const uint32_t total = static_cast<uint32_t>(tiles_m) * tiles_n, id = blockIdx.x, per = total >> 3;
        const uint32_t l = id < per * 8 ? (id & 7) * per + (id >> 3) : id;
        const uint32_t strip = l / (8u * tiles_n), first = strip * 8, rows = min(8u, static_cast<uint32_t>(tiles_m) - first), in = l - strip * 8u * tiles_n;
        tm = static_cast<int>(first + in % rows);
        tn = static_cast<int>(in / rows);
    }
    const int m0 = tm * TILE, n0 = tn * TILE, K = a.K;
    // this thread's chunks of a stage: rows (tid >> 2) + THREADS / 4 * j of w, then of x
    const int row = tid >> 2, chunk = (tid & 3) ^ q8_swizzle(tid >> 2);
    const int8_t* wb = a.w + static_cast<int64_t>(n0) * a.ldw;
    const int8_t* xb = a.x + static_cast<int64_t>(m0) * a.ldx;
    auto row_of = [&](int j) { return j < L / 2 ? min(row + THREADS / 4 * j, a.N - 1 - n0) : min(row + THREADS / 4 * (j - L / 2), a.M - 1 - m0); };   // (past the end: the last one again)
    uint32_t offset[L];
    const int8_t* ptr[L];
#pragma unroll
    for (int j = 0; j < L; ++j) {
        if constexpr (ALIGNED) offset[j] = static_cast<uint32_t>(row_of(j)) * static_cast<uint32_t>(j < L / 2 ? a.ldw : a.ldx) + 16 * chunk;
        else ptr[j] = j < L / 2 ? wb + static_cast<int64_t>(row_of(j)) * a.ldw : xb + static_cast<int64_t>(row_of(j)) * a.ldx;
    }
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) int8_t*)q8_smem));
    auto request_one = [&](int place, const int8_t* from, int j) {   // ALIGNED
        q8_to_lds(from, offset[j], lds0 + (place % kStages) * kStage + wave * 1024 + j * (16 * THREADS));
    };
    auto request = [&](int place, int step) {
#pragma unroll
        for (int j = 0; j < L; ++j) request_one(place, (j < L / 2 ? wb : xb) + static_cast<int64_t>(step) * kStep, j);
    };
    i32x4 reg[ALIGNED ? 1 : L];
    auto fetch = [&](int step) {   // not ALIGNED
        const int k = step * kStep + 16 * chunk;
        if (step < K / kStep) {
#pragma unroll
            for (int j = 0; j < L; ++j) __builtin_memcpy(&reg[j], ptr[j] + k, 16);
        } else {
#pragma unroll
            for (int j = 0; j < L; ++j) reg[j] = q8_load(ptr[j], k, K);
        }
    };
    auto put = [&](int step) {
#pragma unroll
        for (int j = 0; j < L; ++j) *reinterpret_cast<i32x4*>(q8_smem + (step % kStages) * kStage + j * (16 * THREADS) + tid * 16) = reg[j];
    };
    // reads: rows 32 i + lane % 32 of this wavefront's part, chunks 2 h and 2 h + 1
    const int lr = lane & 31, lc = lane >> 5, wn = (wave >> 1) * (TILE / WN), wm = (wave & 1) * (TILE / 2);
    const int sw = q8_swizzle(lr);
    const int at_w = (wn + lr) * kStep, at_x = kHalf + (wm + lr) * kStep;
    i32x4 wf[2][FW], xf[2][FX];
    auto read_one = [&](int step, int h, int q) {
        const int8_t* st = q8_smem + (step % kStages) * kStage + 16 * ((2 * h + lc) ^ sw);
        const int i = q < FW ? q : q - FW;
        (q < FW ? wf[h][i % FW] : xf[h][i % FX]) = *reinterpret_cast<const i32x4*>(st + (q < FW ? at_w : at_x) + i * 32 * kStep);
    };
    auto read = [&](int step, int h) {
#pragma unroll
        for (int q = 0; q < FW + FX; ++q) read_one(step, h, q);
    };
    i32x16 acc[FW][FX];
#pragma unroll
    for (int i = 0; i < FW; ++i)
#pragma unroll
        for (int j = 0; j < FX; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
    // The products of half step h, and between them the reads of the next half step (issued during the first half of the products) and the requests of a later
    // stage (during the second): a wavefront issues in order, and what it issues in one go it does not multiply meanwhile.
    auto multiply = [&](int h, auto&& read_q, auto&& request_j) {
#pragma unroll
        for (int n = 0; n < FW * FX; ++n) {
            acc[n / FX][n % FX] = q8_mma(wf[h][n / FX], xf[h][n % FX], acc[n / FX][n % FX]);
#pragma unroll
            for (int q = 0; q < FW + FX; ++q)
                if (q * FW * FX / (2 * (FW + FX)) == n) read_q(q);
#pragma unroll
            for (int j = 0; j < L; ++j)
                if (j * FW * FX / L == n) request_j(j);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto nothing = [](int) {};
    // ALIGNED: pairs of whole steps through LDS directly, the rest through registers, which cut it off at K
    static_assert(kStages == 4, "two pairs of steps");
    const int steps = ALIGNED ? K / (2 * kStep) * 2 : (K + kStep - 1) / kStep;
    if (steps > 0) {
        if constexpr (ALIGNED) {
            // Two steps at a time: what they need of a row is one cache line, requested as a whole.  One loop without branches: the last steps request the last stage again, and
            // read what nobody uses, so that the number of loads in flight is the same in all.
#pragma unroll
            for (int s = 0; s < kStages; ++s) request(s, min(s & ~1, steps - 2) + (s & 1));
            q8_wait<(kStages - 1) * L>();
            read(0, 0);
            for (int s = 0; s < steps; s += 2) {
                multiply(0, [&](int q) { read_one(s, 1, q); }, nothing);
                q8_wait<2 * L>();
                multiply(1, [&](int q) { read_one(s + 1, 0, q); }, nothing);
                multiply(0, [&](int q) { read_one(s + 1, 1, q); }, nothing);
                q8_wait<0>();   // (the two steps' loads alternate: the next step's are not complete before the one's after it)
                const int64_t next = static_cast<int64_t>(min(s + 4, steps - 2)) * kStep;   // (stages s + 4 and s + 5 take the places of s and s + 1)
                multiply(1, [&](int q) { read_one(s + 2, 0, q); }, [&](int j) {
                    request_one(s, (j < L / 2 ? wb : xb) + next, j);
                    request_one(s + 1, (j < L / 2 ? wb : xb) + next + kStep, j);
                });
            }
            q8_wait<0>();
        } else {
            for (int s = 0; s < kStages - 1; ++s)
                if (s < steps) { fetch(s); put(s); }
            if (kStages - 1 < steps) fetch(kStages - 1);
            __syncthreads();
            read(0, 0);
            for (int s = 0; s < steps; ++s) {
                multiply(0, [&](int q) { read_one(s, 1, q); }, nothing);
                if (s + kStages - 1 < steps) put(s + kStages - 1);
                __syncthreads();
                if (s + kStages < steps) fetch(s + kStages);
                multiply(1, [&](int q) { read_one(s + 1, 0, q); }, nothing);   // (behind the last step: what nobody uses)
            }
        }
    }
    if constexpr (ALIGNED) {
        for (int k = steps * kStep; k < K; k += kStep) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < L; ++j) {
                const int8_t* p = (j < L / 2 ? wb + static_cast<int64_t>(row_of(j)) * a.ldw : xb + static_cast<int64_t>(row_of(j)) * a.ldx);
                *reinterpret_cast<i32x4*>(q8_smem + j * (16 * THREADS) + tid * 16) = q8_load(p, k + 16 * chunk, K);
            }
            __syncthreads();
            read(0, 0); read(0, 1);
            multiply(0, nothing, nothing); multiply(1, nothing, nothing);
        }
    }
    float sx[FX];
#pragma unroll
    for (int j = 0; j < FX; ++j) sx[j] = a.sx[min(m0 + wm + 32 * j + lr, a.M - 1)];
#pragma unroll
    for (int i = 0; i < FW; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const Q8Columns c = q8_columns(a, n0 + wn + 32 * i + 8 * g + 4 * lc);
#pragma unroll
            for (int j = 0; j < FX; ++j)
                q8_store<T>(a, c, m0 + wm + 32 * j + lr, sx[j], acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
        }
}

template <typename T, int TILE, int THREADS, bool ALIGNED> static int launch_tile(const Q8Args& a, hipStream_t st)
{
    constexpr int smem = 2 * TILE * kStep * kStages;
    DQN_HIP(raise_dynamic_lds(reinterpret_cast<const void*>(q8_tile_kernel<T, TILE, THREADS, ALIGNED>), smem));
    const int tm = (a.M + TILE - 1) / TILE, tn = (a.N + TILE - 1) / TILE;
    hipLaunchKernelGGL((q8_tile_kernel<T, TILE, THREADS, ALIGNED>), dim3(static_cast<unsigned>(tm) * tn), dim3(THREADS), smem, st, a, tm, tn);
    DQN_LAUNCH_CHECK();
    return DQN_OK;
}

template <typename T> static int launch_linear(const Q8Args& a, hipStream_t st)
{
    const auto blocks = [&](int bn, int bm) { return dim3(static_cast<unsigned>((a.N + bn - 1) / bn), static_cast<unsigned>((a.M + bm - 1) / bm)); };
    const auto tiles = [&](int64_t t) { return (a.M + t - 1) / t * ((a.N + t - 1) / t); };
    // Streamed: up to 16 rows of x, and while there are no more pieces of 32 than compute units (32 / tiles of 64, in us: 512x512 1024 6.0 / 6.5, 3136 7.8 / 10.8, 8192 18.9 / 31.7; 32x8000
    // 3136 7.7 / 10.7; 512x576 1024 9.5 / 6.3, 3136 13.0 / 10.8, 8192 34.7 / 31.8).  In pieces of 16 while there are few of 32 (16 / 32: 128x512x3136 4.2 / 6.8, 128x1024x3136 6.6 / 7.5,
    // 200x300x16384 17.5 / 31.6, 352x512 k 512 4.3 / 5.0 and 3136 8.4 / 7.6, 384x512x3136 8.5 / 7.5).  A short k has four wavefronts, a longer one eight (4 / 8: 1x65536 k 1024
    // 13.3 / 18.6, 3136 30.4 / 33.7, 4096 48.8 / 46.0; 1x16384 k 3600 11.2 / 11.5, 4096 15.4 / 13.8, 8192 24.9 / 23.7; 8x512x3136 alike).
    if (a.M <= 16 || tiles(32) <= 256) {
        const bool by_16 = a.M <= 16 || tiles(32) < 192;
        if (by_16 && a.K < 4096) hipLaunchKernelGGL((q8_stream_kernel<T, 16, 4, 4>), blocks(16, 16), dim3(256), 0, st, a);
        else if (by_16) hipLaunchKernelGGL((q8_stream_kernel<T, 16, 4, 8>), blocks(16, 16), dim3(512), 0, st, a);
        else hipLaunchKernelGGL((q8_stream_kernel<T, 32, 8, 8>), blocks(32, 32), dim3(512), 0, st, a);
        DQN_LAUNCH_CHECK();
        return DQN_OK;
    }
    // 16-byte loads straight into LDS need rows on 16-byte borders; a lane's place within a tile is a 32-bit offset
    const bool aligned = aligned16(a.x) && aligned16(a.w) && a.ldx % 16 == 0 && a.ldw % 16 == 0 && a.ldx < (1 << 23) && a.ldw < (1 << 23);
    // The largest tile of which there are enough: a smaller one reads its operands more often, a larger one leaves compute units idle (64 / 128, in us: 1024^3 8.1 / 11.6, 1111x2051x2003 20 / 24,
    // 1536x2048x2048 16 / 19, 1792x1792x2048 19.6 / 18.6, 2048^3 20.4 / 18.0, 256x16384x4096 35 / 33).  One of 256 starts and ends slower, which a long k makes up for (128 / 256 on the same
    // aligned operands: 8192x8192 k 1024 111 / 149, 4096 295 / 301, 8192 542 / 500; 4096x4096 k 4096 80 / 85, 8192 141 / 137, 16384 266 / 240; 3328x3328 k 4096 66 / 64, 8192 113 / 105).
    if (tiles(128) < 200) return aligned ? launch_tile<T, 64, 256, true>(a, st) : launch_tile<T, 64, 256, false>(a, st);
    if (tiles(256) < 160 || a.K < 6144) return aligned ? launch_tile<T, 128, 256, true>(a, st) : launch_tile<T, 128, 256, false>(a, st);
    return aligned ? launch_tile<T, 256, 512, true>(a, st) : launch_tile<T, 128, 256, false>(a, st);
}

int enqueue_q8_linear(const int8_t* x, int64_t ldx, const float* sx, const int8_t* w, int64_t ldw, const float* sw, const float* bias, bool relu, int64_t M,
                      int64_t N, int64_t K, void* y, int32_t type, int64_t ldy, hipStream_t st)
{
    const Q8Args a{x, w, sx, sw, bias, y, ldx, ldw, ldy, static_cast<int>(M), static_cast<int>(N), static_cast<int>(K), relu};
    return type == DQN_TYPE_FP32 ? launch_linear<float>(a, st) : type == DQN_TYPE_BF16 ? launch_linear<bf16_t>(a, st) : launch_linear<_Float16>(a, st);
}

}  // namespace dqn

using namespace dqn;

extern "C" {

int q8_quantize_rows(const void* x, int32_t type, int64_t ldx, int64_t rows, int64_t cols, int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv,
                     void* stream)
{
    const char* who = "q8_quantize_rows";
    if (int rc = check_type(who, type)) return rc;
    if (rows < 0 || rows > Q8_QUANTIZE_MAX_ROWS || cols < 0 || cols > Q8_QUANTIZE_MAX_COLS) return fail(DQN_EINVAL, "%s: rows = %lld, cols = %lld", who, (long long)rows, (long long)cols);
    if (rows == 0) return DQN_OK;
    if (!scale || (cols && (!x || (!q && !values)))) return fail(DQN_EINVAL, "%s: null pointer", who);
    const uintptr_t e = type == DQN_TYPE_FP32 ? 4 : 2;
    if (!aligned_to(x, e) || !aligned_to(values, e) || !aligned_to(scale, 4)) return fail(DQN_EINVAL, "%s: a pointer is not aligned to its elements", who);
    if (ldx < cols || (q && ldq < cols) || (values && ldv < cols)) return fail(DQN_EINVAL, "%s: a row pitch is shorter than a row", who);
    hipStream_t st;
    if (int rc = check_stream(who, stream, &st)) return rc;
    return enqueue_quantize_rows(x, type, ldx, rows, cols, q, ldq, scale, values, ldv, st);
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
    hipStream_t st;
    if (int rc = check_stream(who, stream, &st)) return rc;
    return enqueue_q8_linear(x, ldx, sx, w, ldw, sw, bias, relu != 0, M, N, K, y, type, ldy, st);
}

}  // extern "C"
