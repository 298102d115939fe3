// Drawing an index from a row of scores under temperature, top-k, top-p and min-p (include/dqn_mi355.h: policy_sample).
#include <type_traits>

#include "policy.h"
#include "quant.h"

#include "gemm_mfma.h"

namespace dqn {

// ---- weights ------------------------------------------------------------------------------------------------------------
//
// w = exp((x - m) / T) in fp64 and, for every sum, as a whole multiple of 2^-40: sums of whole numbers are the same in any order
// (histograms are filled by atomics, rows are shared out among threads), and with n <= 2^22 they fit 63 bits.
constexpr double kUnits = 0x1p40;

struct RowSettings {
    double t, p, min_p, u;
    int k;         // 0: off
    bool bad, greedy;
};
__device__ inline RowSettings row_settings(const PolicyArgs& a, int64_t row)
{
    RowSettings s;
    const float t = a.temperature ? a.temperature[row] : 1.f, p = a.top_p ? a.top_p[row] : 1.f, mp = a.min_p ? a.min_p[row] : 0.f;
    const float u = a.u ? a.u[row] : static_cast<float>(philox_draw(a.seed, kTagPolicy, a.step, static_cast<uint32_t>(row)).x[0] >> 8) * 0x1p-24f;
    const int k = a.top_k ? a.top_k[row] : 0;
    s.bad = !(t >= 0.f && t < INFINITY) || p != p || mp != mp || u != u;
    s.greedy = t == 0.f || k == 1 || p <= 0.f;
    s.t = t; s.p = p; s.min_p = fmin(static_cast<double>(mp), 1.0);
    s.u = fmin(fmax(static_cast<double>(u), 0.0), 1.0 - 0x1p-24);
    s.k = k > 0 && k < a.n ? k : 0;
    return s;
}

// The score as a whole number that orders as the scores do (-0 and +0 are one value; NaN has been ruled out).
__device__ inline uint32_t score_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float key_score(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// A score with its place: descending order of these is the order of the filters (score descending, index ascending).
__device__ inline uint64_t entry_of(float x, int index) { return static_cast<uint64_t>(score_key(x)) << 32 | static_cast<uint32_t>(~index); }
__device__ inline float entry_score(uint64_t e) { return key_score(static_cast<uint32_t>(e >> 32)); }
__device__ inline int entry_index(uint64_t e) { return static_cast<int>(~static_cast<uint32_t>(e)); }

// a * b + c with c in scalar registers: left to itself the compiler copies each coefficient into vector registers first, two more instructions for each.
__device__ __forceinline__ double fma_s(double a, double b, double c)
{
    double r;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "s"(c));
    return r;
}
template <typename T> __device__ __forceinline__ T uniform(T v)   // the same in every lane: into scalar registers
{
    constexpr int N = sizeof(T) / 4;
    uint32_t w[N];
    __builtin_memcpy(w, &v, sizeof(T));
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = __builtin_amdgcn_readfirstlane(w[i]);
    __builtin_memcpy(&v, w, sizeof(T));
    return v;
}

struct Weights {
    double m, c;   // the row's maximum, log2(e) / T.  Where the maximum is +infinity it counts as 10^39 and c as 10^300: its equals have weight 1, all others 0
    // 2^40 w before it is rounded to a whole number: 2^y = 2^i 2^f, |f| <= 1/2, the second factor by its Taylor series up to f^11 (off by less than 2^-46).
    // Minus infinity and everything far below the maximum end as 2^-960, which is 0 units.
    __device__ __forceinline__ double raw(float x) const
    {
        constexpr double L = 0.693147180559945309417232121458, L2 = L * L / 2, L3 = L2 * L / 3, L4 = L3 * L / 4, L5 = L4 * L / 5, L6 = L5 * L / 6, L7 = L6 * L / 7,
                         L8 = L7 * L / 8, L9 = L8 * L / 9, L10 = L9 * L / 10, L11 = L10 * L / 11, U = kUnits, kRound = 0x1.8p52;   // (adding kRound leaves the nearest whole number in the low bits)
        const double y = fmax((fmin(static_cast<double>(x), 1e39) - m) * c, -1000.0), at = y + kRound, f = y - (at - kRound);
        double v = fma_s(f, uniform(L11 * U), L10 * U);
        v = fma_s(v, f, L9 * U); v = fma_s(v, f, L8 * U); v = fma_s(v, f, L7 * U); v = fma_s(v, f, L6 * U); v = fma_s(v, f, L5 * U);
        v = fma_s(v, f, L4 * U); v = fma_s(v, f, L3 * U); v = fma_s(v, f, L2 * U); v = fma_s(v, f, L * U); v = fma_s(v, f, U);
        const uint64_t bits = __builtin_bit_cast(uint64_t, v);
        const uint32_t i = static_cast<uint32_t>(__builtin_bit_cast(uint64_t, at));
        return __builtin_bit_cast(double, bits + (static_cast<uint64_t>(i << 20) << 32));
    }
    __device__ __forceinline__ double whole(float x) const { return rint(raw(x)); }   // (sums of up to 2^13 of them are exact in fp64; a thread has at most 2^12)
    __device__ __forceinline__ uint64_t units(float x) const { return whole_units(whole(x)); }
    __device__ __forceinline__ static uint64_t whole_units(double w) { return __builtin_bit_cast(uint64_t, w + 0x1p52) - 0x4330000000000000ull; }   // a whole number below 2^52
};
__device__ inline Weights make_weights(float m, double t)
{
    return uniform(m == INFINITY ? Weights{1e39, 1e300} : Weights{m, 1.4426950408889634074 / t});
}

__device__ inline float log_probability(float x, const Weights& w, double t, uint64_t total)
{
    const double d = x == INFINITY ? 0.0 : (static_cast<double>(x) - w.m) / t;
    return static_cast<float>(d - log(static_cast<double>(total) / kUnits));
}
__device__ inline void answer(const PolicyArgs& a, int64_t row, int32_t index, float logp)
{
    a.index[row] = index;
    if (a.logp) a.logp[row] = logp;
}
__device__ inline float not_a_number() { return __uint_as_float(0x7FC00000u); }

__device__ inline uint64_t wave_sum(uint64_t v)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ inline uint64_t wave_scan(uint64_t v)   // inclusive
{
    const int lane = threadIdx.x & 63;
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// ---- short rows: a wavefront each, a lane for each score -------------------------------------------------------------------------
//
// What lies before an entry in the filters' order is counted and summed against all n others (n <= 64), so nothing is sorted.
__device__ __forceinline__ void short_row(const PolicyArgs& a, int64_t row, float x)   // x: this lane's score, -infinity where there is none
{
    const int lane = threadIdx.x & 63;
    const RowSettings s = row_settings(a, row);
    const bool nan = __any(x != x);
    float m = x;
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (s.bad || nan || m == -INFINITY) {
        if (lane == 0) answer(a, row, -1, not_a_number());
        return;
    }
    if (s.greedy) {
        const int first = __builtin_ctzll(__ballot(x == m));
        if (lane == 0) answer(a, row, first, 0.f);
        return;
    }
    const Weights w = make_weights(m, s.t);
    const double raw = w.raw(x);
    const uint64_t mine = static_cast<uint64_t>(rint(raw));
    bool keep = x > -INFINITY;
    if (s.k || s.p < 1.0) {
        const uint64_t e = entry_of(x, lane);
        uint64_t before = 0;
        int rank = 0;
        for (int j = 0; j < a.n; ++j) {
            const uint64_t o = __shfl(e, j), ow = __shfl(mine, j);
            if (o > e) { ++rank; before += ow; }
        }
        if (s.k) keep = keep && rank < s.k;
        if (s.p < 1.0) {
            const double mass = static_cast<double>(wave_sum(keep ? mine : 0));
            keep = keep && (rank == 0 || static_cast<double>(before) < s.p * mass);
        }
    }
    keep = keep && raw >= s.min_p * kUnits;
    const uint64_t sum = wave_scan(keep ? mine : 0), total = __shfl(sum, 63);
    const uint64_t target = static_cast<uint64_t>(s.u * static_cast<double>(total));
    const int pick = __builtin_ctzll(__ballot(sum > target));   // (total is at least 2^40 and u is below 1)
    if (lane == pick) answer(a, row, pick, log_probability(x, w, s.t, total));
}

template <typename T>
__global__ __launch_bounds__(256) void policy_short_kernel(PolicyArgs a, int64_t rows)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = blockIdx.x * 4ll + (threadIdx.x >> 6);
    if (row >= rows) return;
    short_row(a, row, lane < a.n ? static_cast<float>(static_cast<const T*>(a.scores)[row * a.ld + lane]) : -INFINITY);
}

// A workgroup per row: two hidden values per thread become levels in LDS, eight threads sum the products of one action, the first wavefront draws.  Nothing but the chain of launches bounds
// a call this small, and this is one instead of three (act step of 8 states, bf16: 25 us with three, 17 to 20 with one, from run to run: the host's share of its launches).
__global__ __launch_bounds__(256) void policy_q8_head_kernel(PolicyArgs a, const float* hidden, const int8_t* w, const float* scales, const float* bias, const uint64_t* made, const uint64_t* now,
                                                              float* q)
{
    __shared__ uint32_t part[4];
    __shared__ alignas(16) int8_t levels[512];
    __shared__ float scores[32];
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x;
    const bool current = *made == *now;   // else the row's scale is NaN, and with it all that follows
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 h = reinterpret_cast<const f32x2*>(hidden + row * 512)[t];
    uint32_t top = max(magnitude(h[0]), magnitude(h[1]));
    for (int d = 32; d; d >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), d)));
    if ((t & 63) == 0) part[t >> 6] = top;
    __syncthreads();
    top = max(max(part[0], part[1]), max(part[2], part[3]));
    const bool finite = top < 0x7F800000u;
    const float m = finite ? __uint_as_float(top) : 0.f, s = finite && current ? row_scale(m) : not_a_number();
    const Levels l = make_levels(m);
    levels[2 * t] = static_cast<int8_t>(finite ? level_of(l, h[0]) : 0);
    levels[2 * t + 1] = static_cast<int8_t>(finite ? level_of(l, h[1]) : 0);
    __syncthreads();
    const int action = t >> 3, k = (t & 7) * 64;
    int32_t acc = 0;
    if (action < a.n) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const i32x4 v = *reinterpret_cast<const i32x4*>(w + action * 512 + k + 16 * i), x = *reinterpret_cast<const i32x4*>(levels + k + 16 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_sdot4(v[e], x[e], acc, false);
        }
    }
    for (int d = 4; d; d >>= 1) acc += __shfl_xor(acc, d);
    if ((t & 7) == 0 && action < a.n) {
        const float v = q8_result<float>(acc, s, scales[action], bias[action], -INFINITY);
        scores[action] = v;
        q[row * a.n + action] = v;
    }
    __syncthreads();
    if (t < 64) short_row(a, row, t < a.n ? scores[t] : -INFINITY);
}

// ---- longer rows: what the kernels below share ------------------------------------------------------------------------------
//
// The kept set is a prefix of the filters' order cut by min-p, so all a filter has to find is its last entry (a score with its index).
//   top-k with a small k   the k-th largest of some 256 groups' maxima is a lower bound for the k-th largest score: the few entries from it on go into
//                          a list, which is sorted; everything else happens in the list.
//   otherwise              a histogram (mass and, for top-k, entries) of the scores that have mass over BINS equal parts of their range finds the part
//                          in which a count or a mass crosses; its entries go into the list, which is sorted.
// Where the entries overflow the list (equal scores) or there is no range, the crossing is found digit by digit in the scores' keys.
//
// Every pass reads the scores again, from cache: held in registers, they need code without loops, of which the passes over 128 scores per thread took
// 300 KB.  A wavefront has a contiguous stretch, so that the draw, a search in index order, goes from a quarter of such a stretch to one score.  What
// bounds it are the exponentials: 25 instructions at fp64's rate for each.
constexpr int kListK = 192, kPolicyGroups = 512;
// The largest k for which the groups' way is taken.  The nearer k comes to the number of groups, the lower its bound and the longer its list; what it saves is a pass over the row with
// exponentials.  Groups / range, in us, 64 rows: 1000 scores k = 48 13 / 13, 96 19 / 13; 4096: 64 16 / 16, 96 21 / 17; 8192: 80 21 / 21, 128 26 / 21; 16384: 128 28 / 31 (bf16; fp32 27 / 35),
// 160 33 / 31; 32768: 192 38 / 43; 256 rows of 131072: 192 60 / 87 (fp32 83 / 119).
__device__ inline int list_most(int n) { return min(kListK, 48 + n / 192); }

// (sized by the threads: four workgroups of 256 threads fit a compute unit)
template <int THREADS> struct RowShared {
    static constexpr int BINS = 2 * THREADS, LIST = 2 * THREADS;
    alignas(16) uint64_t mass[BINS];   // the histogram
    uint32_t entries[BINS];
    alignas(16) uint64_t list[LIST];
    uint64_t sorted[LIST];
    uint64_t part[16], part2[16];
    alignas(16) uint32_t group[kPolicyGroups];
    uint32_t count;             // entries in the list
    int pick;
    uint64_t pick_sum, bound;
};

template <typename T, int THREADS> struct Row {
    static constexpr int E = 16 / sizeof(T), WAVES = THREADS / 64;
    typedef T vec __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    const T* x;
    int n, trips, lane, wave;
    // the n scores of the row from `from` on; indices count from there
    __device__ Row(const PolicyArgs& a, int64_t row, int from, int n_)
        : x(static_cast<const T*>(a.scores) + row * a.ld + from), n(n_), trips(((n_ + E - 1) / E + THREADS - 1) / THREADS), lane(threadIdx.x & 63),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6))
    {
    }
    __device__ int first(int i) const { return ((wave * trips + i) * 64 + lane) * E; }   // index of the first score of trip i
    __device__ __forceinline__ vec load(int i) const
    {
        const int at = first(i);
        vec v;
        if (at + E <= n) return *reinterpret_cast<const vec*>(x + at);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = at + e < n ? x[at + e] : static_cast<T>(-INFINITY);
        return v;
    }
    // f(index of the first, 16 bytes of scores) for every trip; behind the end they are -infinity.  AHEAD loads are in flight: a pass that hardly
    // computes waits for nothing else, one with exponentials has the other wavefronts to hide a single one.
    template <int AHEAD, typename F> __device__ __forceinline__ void each(const F& f) const
    {
        if constexpr (AHEAD == 1) {
            vec next = load(0);
#pragma unroll 1
            for (int i = 0; i < trips; ++i) {
                const vec v = next;
                if (i + 1 < trips) next = load(i + 1);
                f(first(i), v);
            }
        } else {
            int i = 0;
#pragma unroll 1
            for (; i + AHEAD <= trips; i += AHEAD) {
                vec v[AHEAD];
#pragma unroll
                for (int q = 0; q < AHEAD; ++q) v[q] = load(i + q);
#pragma unroll
                for (int q = 0; q < AHEAD; ++q) f(first(i + q), v[q]);
            }
#pragma unroll 1
            for (; i < trips; ++i) f(first(i), load(i));
        }
    }
    static __device__ __forceinline__ bool any(vec v, float bound)   // of the wavefront's scores is as large
    {
        bool a = false;
#pragma unroll
        for (int e = 0; e < E; ++e) a |= static_cast<float>(v[e]) >= bound;
        return __any(a);
    }
    // f(score, index)
    template <typename F> __device__ __forceinline__ void each_score(const F& f) const
    {
        each<1>([&](int at, const vec& v) {
#pragma unroll
            for (int e = 0; e < E; ++e) f(static_cast<float>(v[e]), at + e);
        });
    }
};

// Sum over the workgroup, to every thread.
template <int WAVES> __device__ inline uint64_t block_sum(uint64_t* part, uint64_t v)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    uint64_t s = 0;
    for (int q = 0; q < WAVES; ++q) s += part[q];
    return s;
}

// The first j of 0 .. BINS - 1 (each thread's are next to each other) at which above + f(0) + .. + f(j) reaches target, and the sum before it.  One
// does, or sh.pick stays -1.
template <int THREADS, typename F> __device__ __forceinline__ void first_reaching(RowShared<THREADS>& sh, const F& f, uint64_t above, double target)
{
    constexpr int PER = RowShared<THREADS>::BINS / THREADS, WAVES = THREADS / 64;
    const int t = threadIdx.x;
    uint64_t v[PER], mine = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) { v[j] = f(t * PER + j); mine += v[j]; }
    const uint64_t upto = wave_scan(mine);
    __syncthreads();
    if (t == 0) sh.pick = -1;
    if ((t & 63) == 63) sh.part[t >> 6] = upto;
    __syncthreads();
    uint64_t sum = above + upto - mine;
    for (int q = 0; q < WAVES; ++q) sum += q < (t >> 6) ? sh.part[q] : 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (static_cast<double>(sum) < target && static_cast<double>(sum + v[j]) >= target) { sh.pick = t * PER + j; sh.pick_sum = sum; }
        sum += v[j];
    }
    __syncthreads();
}

// The entries that `want` takes into a list, in any order, their indices shifted by `offset`; *count goes on beyond LIST where they do not fit.
template <int LIST, typename ROW, typename F> __device__ __forceinline__ void gather(uint64_t* list, uint32_t* count, const ROW& row, int offset, const F& want)
{
    row.template each<4>([&](int first, const typename ROW::vec& v) {
        uint32_t hits = 0;
#pragma unroll
        for (int e = 0; e < ROW::E; ++e) hits |= first + e < row.n && want(static_cast<float>(v[e])) ? 1u << e : 0u;
        if (hits) {   // rare
            uint32_t at = atomicAdd(count, static_cast<uint32_t>(__popc(hits)));
#pragma unroll
            for (int e = 0; e < ROW::E; ++e)
                if (hits >> e & 1) {
                    if (at < LIST) list[at] = entry_of(static_cast<float>(v[e]), offset + first + e);
                    ++at;
                }
        }
    });
}

// sh.list[0 .. count) into sh.sorted[0 .. count), descending.  Up to 256 entries each finds its place by counting the larger ones; more go through a
// bitonic network.
template <int THREADS> __device__ __forceinline__ void sort_list(RowShared<THREADS>& sh, int count)
{
    const int t = threadIdx.x;
    __syncthreads();
    if (count <= 256) {
        if (t < 8 && count + t < 264) sh.list[count + t] = 0;   // (LIST is 512 or more)
        __syncthreads();
        if (t < count) {
            const uint64_t e = sh.list[t];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < count; j += 2) {
                const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(&sh.list[j]);
                rank += (o.x > e) + (o.y > e);
            }
            sh.sorted[rank] = e;
        }
        __syncthreads();
        return;
    }
    int size = 512;   // (at most LIST)
    while (size < count) size <<= 1;
    for (int j = t; j < size; j += THREADS) sh.sorted[j] = j < count ? sh.list[j] : 0;   // (no entry is 0: that is a NaN's key)
    for (int width = 2; width <= size; width <<= 1)
        for (int d = width >> 1; d; d >>= 1) {
            __syncthreads();
            for (int q = t; q < size / 2; q += THREADS) {
                const int lo = (q & ~(d - 1)) * 2 + (q & (d - 1)), hi = lo + d;
                const uint64_t x = sh.sorted[lo], y = sh.sorted[hi];
                if ((x < y) == ((lo & width) == 0)) { sh.sorted[lo] = y; sh.sorted[hi] = x; }
            }
        }
    __syncthreads();
}

// What is known of a row once its largest and smallest score are.
enum class Way { kRefused, kGreedy, kPlain, kShortList, kRange, kDigits };
struct RowState {
    Weights w;
    float m, lo, per;   // scores in (lo, m] have mass; parts of that range per unit of score
    Way way;
    // (rounding is monotone)
    template <int BINS> __device__ __forceinline__ int bin(float x) const { return min(static_cast<int>((m - x) * per), BINS - 1); }
};
template <int BINS> __device__ inline RowState row_state(const RowSettings& s, float hi, float low, bool nan, int list_k)
{
    RowState st;
    st.m = uniform(hi);
    st.w = make_weights(st.m, s.t);
    // entries below m - 28.5 T round to 0 units: whether a filter keeps them shows in nothing
    st.lo = uniform(fmaxf(low, static_cast<float>(fmax(static_cast<double>(hi) - 28.5 * s.t, -0x1.fffffep127)) - 2e-7f * fabsf(hi)));
    st.per = uniform(fminf(static_cast<float>(BINS) / (st.m - st.lo), 0x1.fffffep127f));
    const bool flat = !(st.lo < st.m) || st.m - st.lo == INFINITY;   // no range to divide
    st.way = s.bad || nan || st.m == -INFINITY ? Way::kRefused : s.greedy ? Way::kGreedy : s.k && s.k <= list_k ? Way::kShortList
           : !s.k && !(s.p < 1.0) ? Way::kPlain : flat ? Way::kDigits : Way::kRange;
    return st;
}

// bf16 scores have few values: all those from 2^-24 to 2^8 and their negatives have a place in a table in LDS, so that a long row needs an exponential per value instead of one per
// score.  Others (rare) are treated one by one.  256 rows of 131072, top-p: 131 -> 103 us, of which the counting takes 12 (first pass 26 us, fp16's without it 14; profiles/policy_row_passes.txt); one compute unit's LDS holds one workgroup then, which a row this long fills anyway.
constexpr int kTablePlaces = 8192;
__device__ __forceinline__ uint32_t table_place(bf16_t x)   // kTablePlaces or more: none
{
    const uint32_t b = __builtin_bit_cast(uint16_t, x), above = (b & 0x7FFFu) - (103u << 7);
    return above < 4096u ? above | (b >> 15) << 12 : 0xFFFFFFFFu;
}
__device__ __forceinline__ float table_score(uint32_t place) { return __uint_as_float((((place & 4095u) + (103u << 7)) | (place >> 12) << 15) << 16); }
template <typename T> __device__ __forceinline__ uint32_t table_place(T) { return 0xFFFFFFFFu; }

// Largest and smallest score and NaN of the stretch to every thread (and, where there is a table, how often each value occurs into it and in *others whether there are others); the maxima of `groups` (a power of two, 4 to 256) groups of threads into group[].
template <int THREADS, typename ROW> __device__ __forceinline__ bool extremes(RowShared<THREADS>& sh, const ROW& row, float* hi_out, float* low_out, uint32_t* group, int groups,
                                                                                  uint32_t* counts = nullptr, bool* others = nullptr)
{
    float hi = -INFINITY, low = INFINITY;
    bool nan = false, no_place = false;
    if (counts) {
        for (int i = threadIdx.x; i < kTablePlaces; i += THREADS) counts[i] = 0;
        __syncthreads();
    }
    row.template each<4>([&](int first, const typename ROW::vec& v) {
        if (counts) {
#pragma unroll
            for (int e = 0; e < ROW::E; ++e) {
                const uint32_t place = table_place(v[e]);
                if (place < kTablePlaces) atomicAdd(&counts[place], 1u);
                else no_place |= static_cast<float>(v[e]) > -INFINITY;   // (minus infinity, also behind the end, has no mass)
            }
        }
#pragma unroll
        for (int e = 0; e < ROW::E; ++e) {
            const float x = static_cast<float>(v[e]);
            nan |= x != x;
            hi = fmaxf(hi, x);
            low = first + e < row.n ? fminf(low, x) : low;
        }
    });
    const int width = THREADS / groups;   // threads of a group
    for (int d = 1; d < 64; d <<= 1) {
        if (d == width && (row.lane & (d - 1)) == 0) group[threadIdx.x / d] = score_key(hi);
        hi = fmaxf(hi, __shfl_xor(hi, d));
        low = fminf(low, __shfl_xor(low, d));
    }
    if (row.lane == 0) { sh.part[row.wave] = score_key(hi); sh.part2[row.wave] = score_key(low); }
    nan = __syncthreads_or(nan);
    if (width >= 64 && static_cast<int>(threadIdx.x) < groups) {
        uint64_t g = 0;
        for (int q = 0; q < width / 64; ++q) g = max(g, sh.part[threadIdx.x * (width / 64) + q]);
        group[threadIdx.x] = static_cast<uint32_t>(g);
    }
    for (int q = 0; q < ROW::WAVES; ++q) { hi = fmaxf(hi, key_score(static_cast<uint32_t>(sh.part[q]))); low = fminf(low, key_score(static_cast<uint32_t>(sh.part2[q]))); }
    *hi_out = hi;
    *low_out = low;
    no_place = __syncthreads_or(no_place);
    if (others) *others = no_place;
    return nan;
}

// How many groups: enough that the entries above the k-th largest maximum are few more than k, few enough to rank (this / always 256, in us: 512 rows of 1000 fp32 scores, k = 20
// 11 / 15, 40 14 / 16, 64 16 / 18; 256 rows of 16384: 20 17 / 19, 64 21 / 22).
__device__ __host__ inline int groups_for(int k) { return k <= 24 ? 64 : k <= 64 ? 128 : 256; }

// The k-th largest of sh.group[0 .. n).
template <int THREADS> __device__ __forceinline__ float kth_group(RowShared<THREADS>& sh, int n, int k)
{
    __syncthreads();
    for (int t = threadIdx.x; t < n; t += THREADS) {
        const uint32_t g = sh.group[t];
        int more = 0, as_many = 0;
#pragma unroll 4
        for (int j = 0; j < n; j += 4) {   // (n is a multiple of 4)
            const uint4 o = *reinterpret_cast<const uint4*>(&sh.group[j]);
            more += (o.x > g) + (o.y > g) + (o.z > g) + (o.w > g);
            as_many += (o.x >= g) + (o.y >= g) + (o.z >= g) + (o.w >= g);
        }
        if (more < k && k <= as_many) sh.bound = g;   // (equals write the same)
    }
    __syncthreads();
    return key_score(static_cast<uint32_t>(sh.bound));
}

// A row whose kept entries are all among the `count` of sh.list, the first s.k of which top-k keeps.
template <int THREADS> __device__ __forceinline__ void draw_from_list(RowShared<THREADS>& sh, const PolicyArgs& a, int64_t r, const RowSettings& s, const Weights& w, int count)
{
    constexpr int WAVES = THREADS / 64;
    const int t = threadIdx.x, wave = t >> 6;
    sort_list<THREADS>(sh, count);
    count = min(count, s.k);
    // thread j has entry j of the order
    const uint64_t e = t < count ? sh.sorted[t] : 0;
    const double raw = t < count ? w.raw(entry_score(e)) : 0.0;
    const uint64_t mine = Weights::whole_units(rint(raw));
    uint64_t upto = wave_scan(mine);
    if ((t & 63) == 63) sh.part[wave] = upto;
    __syncthreads();
    uint64_t mass = 0;
    for (int q = 0; q < WAVES; ++q) { upto += q < wave ? sh.part[q] : 0; mass += sh.part[q]; }
    const bool keep = t < count && (t == 0 || static_cast<double>(upto - mine) < s.p * static_cast<double>(mass) || s.p >= 1.0) && raw >= s.min_p * kUnits;
    const uint64_t total = block_sum<WAVES>(sh.part, keep ? mine : 0);
    if (t < kListK) { sh.list[t] = keep ? e : 0; sh.mass[t] = keep ? mine : 0; }
    __syncthreads();
    if (keep) {
        const uint64_t target = static_cast<uint64_t>(s.u * static_cast<double>(total));
        uint64_t before = 0;   // kept mass of lower indices
#pragma unroll 8
        for (int j = 0; j < count; ++j) before += static_cast<uint32_t>(sh.list[j]) > static_cast<uint32_t>(e) ? sh.mass[j] : 0;   // (a lower index has a larger complement)
        if (before <= target && target < before + mine) answer(a, r, entry_index(e), log_probability(entry_score(e), w, s.t, total));
    }
}

// The histogram of the stretch's scores: mass, entries, or both; from the counts of the values where there are such.
template <int THREADS, typename ROW> __device__ __forceinline__ void fill_histogram(RowShared<THREADS>& sh, const ROW& row, const RowState& st, bool masses, bool entries,
                                                                                          const uint32_t* counts = nullptr, bool others = false)
{
    for (int b = threadIdx.x; b < RowShared<THREADS>::BINS; b += THREADS) { sh.mass[b] = 0; sh.entries[b] = 0; }
    __syncthreads();
    auto add = [&](float x, uint64_t mass, uint32_t count) {
        const int b = st.template bin<RowShared<THREADS>::BINS>(x);
        if (masses) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]), static_cast<unsigned long long>(mass));
        if (entries) atomicAdd(&sh.entries[b], count);
    };
    if (counts) {
        for (int i = threadIdx.x; i < kTablePlaces; i += THREADS) {
            const float x = table_score(i);
            if (counts[i] && x >= st.lo) add(x, counts[i] * st.w.units(x), counts[i]);
        }
        if (others)
            row.template each<1>([&](int, const typename ROW::vec& v) {
#pragma unroll
                for (int e = 0; e < ROW::E; ++e) {
                    const float x = static_cast<float>(v[e]);
                    if (table_place(v[e]) >= kTablePlaces && x >= st.lo) add(x, st.w.units(x), 1u);
                }
            });
        __syncthreads();
        return;
    }
    row.template each<1>([&](int, const typename ROW::vec& v) {
        uint64_t u[ROW::E];
        if (!ROW::any(v, st.lo)) return;
        if (masses)
#pragma unroll
        for (int e = 0; e < ROW::E; ++e) {
            u[e] = st.w.units(static_cast<float>(v[e]));
            asm("" : "+v"(u[e]));   // here and not behind the test below: the exponentials of several scores overlap
        }
#pragma unroll
        for (int e = 0; e < ROW::E; ++e) {
            const float x = static_cast<float>(v[e]);
            if (x >= st.lo) add(x, u[e], 1u);
        }
    });
    __syncthreads();
}

// The entry in sh.sorted[0 .. count) at which the count (or mass) reaches target, given what lies above the list; 0 if none does.  *mass: of the list's entries down to it.
template <int THREADS>
__device__ __forceinline__ uint64_t last_in_list(RowShared<THREADS>& sh, const Weights& w, int count, bool by_mass, uint64_t above, double target, uint64_t* mass)
{
    sort_list<THREADS>(sh, count);
    first_reaching<THREADS>(sh, [&](int j) -> uint64_t { return j >= count ? 0 : by_mass ? w.units(entry_score(sh.sorted[j])) : 1; }, above, target);
    const int b = sh.pick;
    uint64_t sum = 0;
    for (int j = threadIdx.x; j < count; j += THREADS) sum += b >= 0 && j <= b ? w.units(entry_score(sh.sorted[j])) : 0;
    *mass = block_sum<THREADS / 64>(sh.part, sum);
    return b < 0 ? 0 : sh.sorted[b];
}

// The last entry that a filter keeps, in the key's digits: by_mass the first at which the mass reaches `target`, else the first at which the count does.
template <int THREADS, typename ROW> __device__ __forceinline__ uint64_t last_by_digits(RowShared<THREADS>& sh, const ROW& row, const Weights& w, bool by_mass, double target)
{
    constexpr int BINS = RowShared<THREADS>::BINS, BITS = BINS == 2048 ? 11 : 9;
    static_assert(BINS == 1 << BITS, "a digit's values have a bin each");
    uint32_t prefix = 0;
    uint64_t above = 0;
#pragma unroll 1
    for (int shift = 32; shift > 0;) {
        const int bits = min(shift, BITS), had = shift;
        shift -= bits;
        __syncthreads();
        for (int b = threadIdx.x; b < BINS; b += THREADS) sh.mass[b] = 0;
        __syncthreads();
        row.each_score([&](float x, int index) {
            const uint32_t key = score_key(x);
            if (index >= row.n || (had < 32 && key >> had != prefix)) return;
            const uint64_t v = by_mass ? w.units(x) : 1;
            if (v) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[(key >> shift) & ((1u << bits) - 1)]), static_cast<unsigned long long>(v));
        });
        __syncthreads();
        first_reaching<THREADS>(sh, [&](int j) { return sh.mass[BINS - 1 - j]; }, above, target);
        prefix = prefix << bits | static_cast<uint32_t>(BINS - 1 - sh.pick);
        above = sh.pick_sum;
    }
    // among the entries of that score the r-th in index order
    const uint64_t v = by_mass ? w.units(key_score(prefix)) : 1;
    int64_t r = static_cast<int64_t>((target - static_cast<double>(above)) / static_cast<double>(v));
    while (r > 1 && static_cast<double>(above + (r - 1) * v) >= target) --r;
    while (r < 1 || static_cast<double>(above + r * v) < target) ++r;
    // wavefronts own stretches in index order: theirs first, then trips, then lanes
    uint64_t mine = 0;
    row.each_score([&](float x, int index) { mine += index < row.n && score_key(x) == prefix; });
    mine = wave_sum(mine);
    __syncthreads();
    if (row.lane == 0) sh.part2[row.wave] = mine;
    __syncthreads();
    int64_t left = r;
    int owner = -1;
    for (int q = 0; q < ROW::WAVES; ++q) {
        const int64_t c = static_cast<int64_t>(sh.part2[q]);
        if (owner < 0 && left <= c) owner = q;
        if (owner < 0) left -= c;
    }
    if (row.wave == owner) {
        row.template each<1>([&](int first, const typename ROW::vec& v8) {
            uint64_t c = 0;
#pragma unroll
            for (int e = 0; e < ROW::E; ++e) c += first + e < row.n && score_key(static_cast<float>(v8[e])) == prefix;
            const uint64_t upto = wave_scan(c);
            const int64_t before = static_cast<int64_t>(upto - c), all = static_cast<int64_t>(__shfl(upto, 63));
            if (left > 0 && left > before && left <= static_cast<int64_t>(upto)) {
                int64_t need = left - before;
#pragma unroll
                for (int e = 0; e < ROW::E; ++e)
                    if (first + e < row.n && score_key(static_cast<float>(v8[e])) == prefix && --need == 0) sh.bound = entry_of(static_cast<float>(v8[e]), first + e);
            }
            left = left > all ? left - all : 0;
        });
    }
    __syncthreads();
    return sh.bound;
}

// What of a stretch is kept: entries down to `last` (0: all) whose weight min-p allows; `offset` is the index of the stretch's first score.
struct Kept {
    float score;
    int index;
    double min_raw;
    __device__ Kept(uint64_t last, int offset, double min_p) : score(last ? entry_score(last) : -INFINITY), index(last ? entry_index(last) - offset : 0x7FFFFFFF), min_raw(min_p * kUnits) {}
    __device__ __forceinline__ double operator()(const Weights& w, float x, int i) const
    {
        const double raw = w.raw(x);
        const bool in = (x > score) | ((x == score) & (i <= index));
        return (in & (raw >= min_raw)) ? rint(raw) : 0.0;   // (no branches: the exponentials of several scores overlap)
    }
};

// The draw from a stretch.  total: all kept mass of the row and target what is left of u's share of it where the stretch begins; where total is 0, the stretch is the whole row and both are found here.
template <int THREADS, typename ROW>
__device__ __forceinline__ void draw(RowShared<THREADS>& sh, const PolicyArgs& a, int64_t r, const ROW& row, int offset, const RowSettings& s, const Weights& w, uint64_t last, uint64_t total,
                                     uint64_t target, uint64_t* table = nullptr)
{
    constexpr int WAVES = THREADS / 64, E = ROW::E;
    const Kept kept(last, offset, s.min_p);
    const int t = threadIdx.x, per = (row.trips + 3) / 4;
    uint64_t sums[4] = {0, 0, 0, 0};   // of four groups of this lane's trips
    if (table) {   // what a score of each value counts, if it is kept
        __syncthreads();
        for (int i = t; i < kTablePlaces; i += THREADS) reinterpret_cast<double*>(table)[i] = kept(w, table_score(i), INT32_MIN);
        __syncthreads();
    }
    {
        double sum = 0.0;
        int left = per, group = 0;
        auto close = [&] {
#pragma unroll
            for (int q = 0; q < 4; ++q) sums[q] = q == group ? Weights::whole_units(sum) : sums[q];
            sum = 0.0;
            left = per;
            ++group;
        };
        if (table) {
            row.template each<4>([&](int first, const typename ROW::vec& v) {
                if (ROW::any(v, kept.score)) {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float x = static_cast<float>(v[e]);
                        if (x > kept.score || (x == kept.score && first + e <= kept.index)) {
                            const uint32_t place = table_place(v[e]);
                            if (place < kTablePlaces) sum += reinterpret_cast<const double*>(table)[place];
                            else if (x > -INFINITY) sum += kept(w, x, first + e);
                        }
                    }
                }
                if (--left == 0) close();
            });
        } else {
            row.template each<1>([&](int first, const typename ROW::vec& v) {
                if (ROW::any(v, kept.score)) {
#pragma unroll
                    for (int e = 0; e < E; ++e) sum += kept(w, static_cast<float>(v[e]), first + e);
                }
                if (--left == 0) close();
            });
        }
        if (left < per) close();
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[q] = wave_sum(sums[q]);
    __syncthreads();
    if (row.lane < 4) sh.mass[row.wave * 4 + row.lane] = row.lane == 0 ? sums[0] : row.lane == 1 ? sums[1] : row.lane == 2 ? sums[2] : sums[3];
    __syncthreads();
    if (total == 0) {
        for (int q = 0; q < 4 * WAVES; ++q) total += sh.mass[q];
        target = static_cast<uint64_t>(s.u * static_cast<double>(total));
    }
    int owner = -1;
    for (int q = 0; q < 4 * WAVES; ++q) {
        if (owner < 0 && target < sh.mass[q]) owner = q;
        if (owner < 0) target -= sh.mass[q];
    }
    if (owner < 0) return;   // (not reached: the kept sums of a stretch are the same whole numbers wherever they are taken)
    // the stretch of that group, shared out among all threads
    const int begin = ((owner >> 2) * row.trips + (owner & 3) * per) * 64 * E, end = min(row.n, ((owner >> 2) * row.trips + min(((owner & 3) + 1) * per, row.trips)) * 64 * E);
    const int each = (end - begin + THREADS - 1) / THREADS, from = begin + t * each, to = min(end, from + each);
    double sum = 0.0;
    for (int i = from; i < to; ++i) sum += kept(w, static_cast<float>(row.x[i]), i);
    const uint64_t own = Weights::whole_units(sum);
    uint64_t upto = wave_scan(own);
    if (row.lane == 63) sh.part[row.wave] = upto;
    __syncthreads();
    for (int q = 0; q < WAVES; ++q) upto += q < row.wave ? sh.part[q] : 0;
    if (target < upto - own || target >= upto) return;
    uint64_t at = upto - own;
    for (int i = from; i < to; ++i) {
        const float x = static_cast<float>(row.x[i]);
        at += Weights::whole_units(kept(w, x, i));
        if (target < at) return answer(a, r, offset + i, log_probability(x, w, s.t, total));
    }
}

// The lowest index of the row's maximum in the stretch, or 2^31 - 1.
template <int THREADS, typename ROW> __device__ __forceinline__ int first_of(RowShared<THREADS>& sh, const ROW& row, float m)
{
    int first = 0x7FFFFFFF;
    row.template each<4>([&](int at, const typename ROW::vec& v) {
#pragma unroll
        for (int e = 0; e < ROW::E; ++e) first = static_cast<float>(v[e]) == m ? min(first, at + e) : first;
    });
    for (int d = 32; d; d >>= 1) first = min(first, __shfl_xor(first, d));
    __syncthreads();
    if (row.lane == 0) sh.part[row.wave] = static_cast<uint64_t>(first);
    __syncthreads();
    for (int q = 0; q < ROW::WAVES; ++q) first = min(first, static_cast<int>(sh.part[q]));
    return first;
}

// ---- a row by one workgroup -----------------------------------------------------------------------------------------------
template <typename T, int THREADS> __device__ __forceinline__ void whole_row(RowShared<THREADS>& sh, const PolicyArgs& a, int64_t r, uint64_t* table)
{
    typedef Row<T, THREADS> ROW;
    const ROW row(a, r, 0, a.n);
    const RowSettings s = row_settings(a, r);
    float hi, low;
    const int groups = groups_for(s.k), list_k = list_most(a.n);
    bool others = false;
    uint32_t* counts = !s.greedy && (s.k > list_k || (!s.k && s.p < 1.0)) ? reinterpret_cast<uint32_t*>(table) : nullptr;   // (for the histogram)
    const bool nan = extremes<THREADS>(sh, row, &hi, &low, sh.group, groups, counts, &others);
    const RowState st = row_state<RowShared<THREADS>::BINS>(s, hi, low, nan, list_k);
    if (st.way == Way::kRefused) {
        if (threadIdx.x == 0) answer(a, r, -1, not_a_number());
        return;
    }
    if (st.way == Way::kGreedy) {
        const int first = first_of(sh, row, st.m);
        if (threadIdx.x == 0) answer(a, r, first, 0.f);
        return;
    }
    if (threadIdx.x == 0) sh.count = 0;
    if (st.way == Way::kShortList) {
        const float bound = kth_group<THREADS>(sh, groups, s.k);
        gather<RowShared<THREADS>::LIST>(sh.list, &sh.count, row, 0, [&](float x) { return x >= bound && x > -INFINITY; });   // (fewer than k finite scores: bound is -infinity)
        __syncthreads();
        if (sh.count <= RowShared<THREADS>::LIST) return draw_from_list<THREADS>(sh, a, r, s, st.w, static_cast<int>(sh.count));
    }
    uint64_t last = 0;
    bool by_digits = st.way == Way::kDigits || st.way == Way::kShortList;
    if (st.way == Way::kRange) {
        fill_histogram<THREADS>(sh, row, st, s.p < 1.0, s.k > 0, counts, others);
        uint64_t kept_mass = 0;   // of what top-k leaves
#pragma unroll 1
        for (int filter = s.k ? 0 : 1; filter < (s.p < 1.0 ? 2 : 1) && !by_digits; ++filter) {
            const bool by_mass = filter == 1;
            if (!s.k || (by_mass && kept_mass == 0)) {   // all of it
                uint64_t sum = 0;
                for (int b = threadIdx.x; b < RowShared<THREADS>::BINS; b += THREADS) sum += sh.mass[b];
                kept_mass = block_sum<THREADS / 64>(sh.part, sum);
            }
            const double target = by_mass ? s.p * static_cast<double>(kept_mass) : s.k;
            first_reaching<THREADS>(sh, [&](int j) -> uint64_t { return by_mass ? sh.mass[j] : sh.entries[j]; }, 0, target);
            const int b = sh.pick;
            const uint64_t above = sh.pick_sum;
            if (b < 0) continue;   // fewer than k have mass: all of them are kept
            uint64_t sum = 0;
            for (int j = threadIdx.x; j < b; j += THREADS) sum += sh.mass[j];
            sum = block_sum<THREADS / 64>(sh.part, sum);
            if (threadIdx.x == 0) sh.count = 0;
            __syncthreads();
            gather<RowShared<THREADS>::LIST>(sh.list, &sh.count, row, 0, [&](float x) { return x >= st.lo && st.template bin<RowShared<THREADS>::BINS>(x) == b; });
            __syncthreads();
            if (sh.count > RowShared<THREADS>::LIST) { by_digits = true; break; }
            uint64_t mass;
            last = last_in_list<THREADS>(sh, st.w, static_cast<int>(sh.count), by_mass, above, target, &mass);
            kept_mass = sum + mass;
        }
    }
    if (by_digits) {
        last = 0;
        const uint64_t floor = st.m == INFINITY ? entry_of(INFINITY, 0x7FFFFFFF) : 0;   // beside +infinity nothing has mass: its last entry, behind every index
#pragma unroll 1
        for (int filter = 0; filter < 2; ++filter) {
            if (filter == 0 ? !s.k : !(s.p < 1.0)) continue;
            double target = s.k;
            if (filter == 1) {
                double sum = 0.0;
                row.each_score([&](float x, int index) {
                    if (x > -INFINITY && entry_of(x, index) >= max(last, floor)) sum += st.w.whole(x);
                });
                target = s.p * static_cast<double>(block_sum<THREADS / 64>(sh.part, Weights::whole_units(sum)));
            }
            last = last_by_digits<THREADS>(sh, row, st.w, filter == 1, target);
        }
        last = max(last, floor);
    }
    draw<THREADS>(sh, a, r, row, 0, s, st.w, last, 0, 0, table);
}

template <typename T, int THREADS> constexpr bool kWithTable = std::is_same<T, bf16_t>::value && THREADS == 1024;

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void policy_row_kernel(PolicyArgs a)
{
    __shared__ RowShared<THREADS> sh;
    extern __shared__ uint64_t policy_table[];   // kTablePlaces, where kWithTable
    whole_row<T, THREADS>(sh, a, blockIdx.x, kWithTable<T, THREADS> ? policy_table : nullptr);
}

// ---- few long rows: a row by several workgroups ------------------------------------------------------------------------------
//
// One compute unit takes 30 to 120 us for a row of 131072, so a few rows are shared out: `parts` workgroups per row, a launch for each point at which they have to
// know of each other (no workgroup waits for another one), and in between a record per row in the caller's workspace.
//   1  extremes, groups' maxima                     2  short list | histogram | kept mass of each part
//   3  draw (short list, no filter) | entries of the part of the range that the last kept one lies in, kept mass above it        4  draw
// A row that the list or the range cannot hold is done by one workgroup in the last launch.
constexpr int kParts = 64, kPartThreads = 1024, kPartMin = 4096;
// (as list_most: one row of 65536, k = 96 31 / 42 us in bf16, 128 43 / 42, 160 56 / 42, where equal scores overflow the list; fp32 128 32 / 42, 160 39 / 42, 192 41 / 42)
constexpr int kPartListK = 128;
typedef RowShared<kPartThreads> PartShared;

struct SplitRow {
    uint64_t mass[PartShared::BINS];
    uint32_t entries[PartShared::BINS];
    uint64_t list[2][PartShared::LIST];
    uint64_t kept[kParts];
    uint32_t hi[kParts], low[kParts], nan[kParts], first[kParts];
    uint32_t group[kPolicyGroups];
    uint32_t count[2];   // entries in the lists: the last kept one is among the second where both filters are on, top-k's border in the first
};

// A launch costs about 4 us, so the rows have to be long, and few: they share the compute units, and from 65 on each has three workgroups at most.  One workgroup per row against this,
// bf16, in us: one row of 32768, temperature alone 28 / 27, top-p 45 / 44, top-k 50 20 / 26; of 49152: 32 / 25, 52 / 43, 23 / 29; of 131072: 51 / 27, 89 / 48, 31 / 26; 64 rows of
// 131072: 54 / 44, 97 / 87, 33 / 33; 72 rows: 54 / 54, 94 / 100, 33 / 39; 128 rows: 54 / 62, 96 / 121, 33 / 38.
struct SplitPlan { int parts, len, groups; };   // len: scores of a part, groups per part
static SplitPlan split_plan(int64_t rows, int64_t n)
{
    SplitPlan p{1, static_cast<int>(n), 0};
    if (rows < 1 || rows > 64 || n < 12 * kPartMin) return p;
    int64_t parts = n / kPartMin;
    if (parts > 256 / rows) parts = 256 / rows;
    if (parts > kParts) parts = kParts;
    p.len = static_cast<int>(((n + parts - 1) / parts + 511) / 512 * 512);
    p.parts = static_cast<int>((n + p.len - 1) / p.len);
    p.groups = 4;
    while (p.groups * p.parts < 256) p.groups *= 2;   // (256 to 511 in all)
    return p;
}

template <typename T, int PHASE>
__global__ __launch_bounds__(kPartThreads) void policy_split_kernel(PolicyArgs a, SplitPlan plan, SplitRow* records, int last_phase)
{
    constexpr int THREADS = kPartThreads, WAVES = THREADS / 64, BINS = PartShared::BINS, LIST = PartShared::LIST;
    typedef Row<T, THREADS> ROW;
    __shared__ PartShared sh;
    const int64_t r = blockIdx.y;
    const int part = blockIdx.x, t = threadIdx.x, from = part * plan.len;
    SplitRow& rec = records[r];
    const ROW row(a, r, from, min(plan.len, a.n - from));
    const RowSettings s = row_settings(a, r);
    if constexpr (PHASE == 1) {
        float hi, low;
        const bool nan = extremes<THREADS>(sh, row, &hi, &low, rec.group + part * plan.groups, plan.groups);
        if (t == 0) { rec.hi[part] = score_key(hi); rec.low[part] = score_key(low); rec.nan[part] = nan; }
        for (int b = part * THREADS + t; b < BINS; b += plan.parts * THREADS) { rec.mass[b] = 0; rec.entries[b] = 0; }
        if (part == 0 && t < 2) rec.count[t] = 0;
        return;
    }
    // every wavefront looks at all parts' extremes
    uint32_t hi = 0, low = 0xFFFFFFFFu;
    bool nan = false;
    if (row.lane < plan.parts) { hi = rec.hi[row.lane]; low = rec.low[row.lane]; nan = rec.nan[row.lane] != 0; }
    for (int d = 32; d; d >>= 1) { hi = max(hi, static_cast<uint32_t>(__shfl_xor(static_cast<int>(hi), d))); low = min(low, static_cast<uint32_t>(__shfl_xor(static_cast<int>(low), d))); }
    nan = __any(nan);
    const RowState st = row_state<BINS>(s, key_score(hi), key_score(low), nan, kPartListK);
    const bool both = s.k && s.p < 1.0;
    // the part that u's share of the kept mass falls into, given all parts' kept mass in sh.mass: its workgroup draws
    auto draw_in_part = [&](uint64_t last) {
        uint64_t total = 0;
        for (int q = 0; q < plan.parts; ++q) total += sh.mass[q];
        uint64_t target = static_cast<uint64_t>(s.u * static_cast<double>(total));
        int owner = -1;
        for (int q = 0; q < plan.parts; ++q) {
            if (owner < 0 && target < sh.mass[q]) owner = q;
            if (owner < 0) target -= sh.mass[q];
        }
        __syncthreads();
        if (owner == part) draw<THREADS>(sh, a, r, row, from, s, st.w, last, total, target);
    };
    if constexpr (PHASE == 2) {
        if (st.way == Way::kGreedy) {
            const int first = first_of(sh, row, st.m);
            if (t == 0) rec.first[part] = first == 0x7FFFFFFF ? 0x7FFFFFFFu : static_cast<uint32_t>(from + first);
        } else if (st.way == Way::kShortList) {
            const int groups = plan.parts * plan.groups;
            for (int g = t; g < groups; g += THREADS) sh.group[g] = rec.group[g];
            const float bound = kth_group<THREADS>(sh, groups, s.k);
            gather<LIST>(rec.list[0], &rec.count[0], row, from, [&](float x) { return x >= bound && x > -INFINITY; });
        } else if (st.way == Way::kRange) {
            fill_histogram<THREADS>(sh, row, st, s.p < 1.0, s.k > 0);
            for (int b = t; b < BINS; b += THREADS) {
                if (sh.mass[b]) atomicAdd(reinterpret_cast<unsigned long long*>(&rec.mass[b]), static_cast<unsigned long long>(sh.mass[b]));
                if (sh.entries[b]) atomicAdd(&rec.entries[b], sh.entries[b]);
            }
        } else if (st.way == Way::kPlain) {
            const Kept kept(0, from, s.min_p);
            double sum = 0.0;
            row.each_score([&](float x, int index) { sum += kept(st.w, x, index); });
            const uint64_t all = block_sum<WAVES>(sh.part, Weights::whole_units(sum));
            if (t == 0) rec.kept[part] = all;
        }
        return;
    }
    // ---- rows that are answered here
    if (PHASE == 3 && (st.way == Way::kRefused || st.way == Way::kGreedy)) {
        if (part != 0 || t != 0) return;
        uint32_t first = 0x7FFFFFFFu;
        if (st.way == Way::kGreedy)
            for (int q = 0; q < plan.parts; ++q) first = min(first, rec.first[q]);
        st.way == Way::kGreedy ? answer(a, r, static_cast<int32_t>(first), 0.f) : answer(a, r, -1, not_a_number());
        return;
    }
    if (PHASE == 3 && st.way == Way::kPlain) {
        if (t < plan.parts) sh.mass[t] = rec.kept[t];
        __syncthreads();
        return draw_in_part(0);
    }
    auto fetch_list = [&](int which) {   // into sh.list; false if it overflowed
        const uint32_t count = rec.count[which];
        if (count > LIST) return false;
        for (uint32_t j = t; j < count; j += THREADS) sh.list[j] = rec.list[which][j];
        return true;
    };
    bool one_workgroup = st.way == Way::kDigits;
    if (st.way == Way::kShortList) {
        one_workgroup = rec.count[0] > LIST;
        if (PHASE == 3 && !one_workgroup && part == 0) {
            fetch_list(0);
            draw_from_list<THREADS>(sh, a, r, s, st.w, static_cast<int>(rec.count[0]));
        }
    }
    if (st.way == Way::kRange) {
        auto border = [&](bool by_mass, double target, uint64_t* above) {   // the part of the range, or -1: all is kept
            first_reaching<THREADS>(sh, [&](int j) -> uint64_t { return by_mass ? rec.mass[j] : rec.entries[j]; }, 0, target);
            *above = sh.pick_sum;
            return sh.pick;
        };
        auto mass_before = [&](int b) {   // of the parts of the range before b
            uint64_t sum = 0;
            for (int j = t; j < b; j += THREADS) sum += rec.mass[j];
            return block_sum<WAVES>(sh.part, sum);
        };
        auto in_range = [&](float x, int b0, int b1) { return x >= st.lo && st.template bin<BINS>(x) >= b0 && st.template bin<BINS>(x) <= b1; };
        uint64_t above, ignored;
        int k_bin = -1, first = 0, second = -1;   // top-k's part of the range (-1: it keeps all); the parts first .. second of the last kept entry (none: all is kept)
        uint64_t k_above = 0, k_mass = 0;
        if (s.k) {
            k_bin = border(false, s.k, &k_above);
            k_mass = mass_before(k_bin < 0 ? BINS : k_bin);
            first = second = k_bin;
            if (k_bin < 0) first = 0;
        } else {
            first = second = border(true, s.p * static_cast<double>(mass_before(BINS)), &ignored);
        }
        if (both) {   // what top-k leaves of its part is not known before its list is: top-p's border between the extremes
            const uint64_t most = k_mass + (k_bin < 0 ? 0 : rec.mass[k_bin]);
            first = max(border(true, s.p * static_cast<double>(k_mass), &ignored), 0);
            second = border(true, s.p * static_cast<double>(most), &ignored);
        }
        const int which = both ? 1 : 0;
        if (PHASE == 3) {
            if (both && k_bin >= 0) gather<LIST>(rec.list[0], &rec.count[0], row, from, [&](float x) { return in_range(x, k_bin, k_bin); });
            if (second >= 0) gather<LIST>(rec.list[which], &rec.count[which], row, from, [&](float x) { return in_range(x, first, second); });
            // kept mass of the part's scores above those
            const Kept kept(0, from, s.min_p);
            const int end = second >= 0 ? first : BINS;
            double sum = 0.0;
            row.template each<1>([&](int at, const typename ROW::vec& v) {
                if (!ROW::any(v, st.lo)) return;
#pragma unroll
                for (int e = 0; e < ROW::E; ++e) {
                    const float x = static_cast<float>(v[e]);
                    const double w = kept(st.w, x, at + e);
                    sum += ((x >= st.lo) & (st.template bin<BINS>(x) < end)) ? w : 0.0;
                }
            });
            const uint64_t all = block_sum<WAVES>(sh.part, Weights::whole_units(sum));
            if (t == 0) rec.kept[part] = all;
        } else {
            one_workgroup = rec.count[0] > LIST || (both && rec.count[1] > LIST);
            if (!one_workgroup) {
                uint64_t last = 0;
                if (both && k_bin >= 0) {
                    uint64_t in_list;
                    fetch_list(0);
                    last = last_in_list<THREADS>(sh, st.w, static_cast<int>(rec.count[0]), false, k_above, s.k, &in_list);
                    k_mass += in_list;
                }
                int count = 0;
                if (second >= 0) {
                    const double target = both ? s.p * static_cast<double>(k_mass) : s.k ? s.k : s.p * static_cast<double>(mass_before(BINS));
                    above = s.k && !both ? k_above : mass_before(first);
                    __syncthreads();
                    fetch_list(which);
                    count = static_cast<int>(rec.count[which]);
                    last = last_in_list<THREADS>(sh, st.w, count, s.p < 1.0, above, target, &ignored);
                }
                if (t < plan.parts) sh.mass[t] = rec.kept[t];
                __syncthreads();
                for (int j = t; j < count; j += THREADS) {   // the list's kept entries, to their parts
                    const uint64_t e = sh.sorted[j];
                    const double raw = st.w.raw(entry_score(e));
                    if (e >= last && raw >= s.min_p * kUnits) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[entry_index(e) / plan.len]), static_cast<unsigned long long>(Weights::whole_units(rint(raw))));
                }
                __syncthreads();
                return draw_in_part(last);
            }
        }
    }
    if (PHASE == last_phase && one_workgroup && part == 0) {
        __syncthreads();
        whole_row<T, THREADS>(sh, a, r, nullptr);
    }
}

template <typename T> static int launch_policy(const PolicyArgs& a, int64_t rows, void* work, hipStream_t st)
{
    const SplitPlan plan = split_plan(rows, a.n);
    const dim3 grid(static_cast<unsigned>(rows));
    if (plan.parts > 1) {
        const int phases = a.top_k || a.top_p ? 4 : 3;
        const dim3 parts(static_cast<unsigned>(plan.parts), static_cast<unsigned>(rows));
        SplitRow* records = static_cast<SplitRow*>(work);
        void (*kernels[4])(PolicyArgs, SplitPlan, SplitRow*, int) = {policy_split_kernel<T, 1>, policy_split_kernel<T, 2>, policy_split_kernel<T, 3>, policy_split_kernel<T, 4>};
        for (int p = 0; p < phases; ++p) {
            hipLaunchKernelGGL(kernels[p], parts, dim3(kPartThreads), 0, st, a, plan, records, phases);
            DQN_LAUNCH_CHECK();
        }
        return DQN_OK;
    }
    // (a workgroup for each row of 64 scores: 512 rows temperature alone 8.4 us, this way 3.7; top-p 14 and 7.7)
    if (a.n <= 64) hipLaunchKernelGGL(policy_short_kernel<T>, dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(256), 0, st, a, rows);
    // Four workgroups of 256 threads fit a compute unit, one of 1024: with more rows than compute units the small ones win up to longer rows.  256 / 1024 threads, in us, temperature
    // alone, top-p, top-k 50; 256 rows fp32: 8192 scores 15 / 23, 26 / 35, 19 / 19; 16384: 20 / 27, 37 / 41, 22 / 21; 24576: 25 / 29, 49 / 47, 24 / 22; bf16 alike (16384: 19 / 28,
    // 38 / 41, 20 / 20).  512 rows fp32: 16384: 25 / 48, 45 / 76, 24 / 37; 32768: 43 / 62, 79 / 103, 36 / 46; bf16: 32768: 37 / 58, 77 / 92, 29 / 41.  Beyond, a border among many scores may
    // overflow the small workgroup's list (49152 Laplace-distributed scores, top-p: 280 / 117).
    else if (a.n <= (rows > 256 ? 32768 : 16384)) hipLaunchKernelGGL((policy_row_kernel<T, 256>), grid, dim3(256), 0, st, a);
    else {
        constexpr int smem = kWithTable<T, 1024> ? kTablePlaces * static_cast<int>(sizeof(uint64_t)) : 0;
        if (smem) DQN_HIP(raise_dynamic_lds(reinterpret_cast<const void*>(policy_row_kernel<T, 1024>), smem));
        hipLaunchKernelGGL((policy_row_kernel<T, 1024>), grid, dim3(1024), smem, st, a);
    }
    DQN_LAUNCH_CHECK();
    return DQN_OK;
}

int enqueue_policy_q8_head(const PolicyArgs& a, const float* hidden, const int8_t* w, const float* scales, const float* bias, const uint64_t* made, const uint64_t* now,
                           float* q, int64_t rows, hipStream_t st)
{
    hipLaunchKernelGGL(policy_q8_head_kernel, dim3(static_cast<unsigned>(rows)), dim3(256), 0, st, a, hidden, w, scales, bias, made, now, q);
    DQN_LAUNCH_CHECK();
    return DQN_OK;
}

int enqueue_policy_sample(const PolicyArgs& a, int32_t type, int64_t rows, void* work, hipStream_t st)
{
    return type == DQN_TYPE_FP32 ? launch_policy<float>(a, rows, work, st) : type == DQN_TYPE_BF16 ? launch_policy<bf16_t>(a, rows, work, st) : launch_policy<_Float16>(a, rows, work, st);
}

}  // namespace dqn

using namespace dqn;

extern "C" {

size_t policy_sample_workspace(int64_t rows, int64_t n)
{
    if (rows < 1 || rows > POLICY_SAMPLE_MAX_ROWS || n < 1 || n > POLICY_SAMPLE_MAX_N || split_plan(rows, n).parts == 1) return 0;
    return static_cast<size_t>(rows) * sizeof(SplitRow);
}

int policy_sample(const void* scores, int32_t type, int64_t ld, int64_t rows, int64_t n, const float* temperature, const int32_t* top_k, const float* top_p,
                  const float* min_p, const float* u, int32_t* index, float* logp, void* work, size_t work_bytes, void* stream)
{
    const char* who = "policy_sample";
    if (int rc = check_type(who, type)) return rc;
    if (rows < 0 || rows > POLICY_SAMPLE_MAX_ROWS || n < 0 || n > POLICY_SAMPLE_MAX_N) return fail(DQN_EINVAL, "%s: rows = %lld, n = %lld", who, (long long)rows, (long long)n);
    if (rows == 0) return DQN_OK;
    if ((n && !scores) || !u || !index) return fail(DQN_EINVAL, "%s: null pointer", who);
    if (!aligned_to(scores, type == DQN_TYPE_FP32 ? 4 : 2) || !aligned_to(temperature, 4) || !aligned_to(top_k, 4) || !aligned_to(top_p, 4) || !aligned_to(min_p, 4) ||
        !aligned_to(u, 4) || !aligned_to(index, 4) || !aligned_to(logp, 4) || !aligned16(work))
        return fail(DQN_EINVAL, "%s: a pointer is not aligned to its elements", who);
    if (ld < n) return fail(DQN_EINVAL, "%s: ld = %lld is shorter than a row of %lld", who, (long long)ld, (long long)n);
    if (const size_t need = policy_sample_workspace(rows, n); need && (!work || work_bytes < need)) return fail(DQN_EINVAL, "%s: work holds %zu bytes, needed %zu", who, work ? work_bytes : 0, need);
    hipStream_t st;
    if (int rc = check_stream(who, stream, &st)) return rc;
    const PolicyArgs a{scores, ld, static_cast<int32_t>(n), temperature, top_k, top_p, min_p, u, 0, 0, index, logp};
    return enqueue_policy_sample(a, type, rows, work, st);
}

}  // extern "C"
