// Drawing an index from a row of scores under temperature, top-k, top-p and min-p (include/dqn_mi355.h: policy_sample).
#include "policy.h"

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

struct Weights {
    double m, c;   // the row's maximum, log2(e) / T
    bool inf;      // m is +infinity: its equals have weight 1, all others 0
    // 2^40 w before it is rounded to a whole number: 2^y = 2^i 2^f, |f| <= 1/2, the second factor by its Taylor series up to f^11 (off by less than 2^-46).
    // Minus infinity and everything far below the maximum end as 2^-1060, which is 0 units.
    __device__ __forceinline__ double raw(float x) const
    {
        if (inf) return x == INFINITY ? kUnits : 0.0;
        constexpr double L = 0.693147180559945309417232121458, L2 = L * L / 2, L3 = L2 * L / 3, L4 = L3 * L / 4, L5 = L4 * L / 5, L6 = L5 * L / 6, L7 = L6 * L / 7,
                         L8 = L7 * L / 8, L9 = L8 * L / 9, L10 = L9 * L / 10, L11 = L10 * L / 11;
        const double y = fmax((static_cast<double>(x) - m) * c, -1100.0), i = rint(y), f = y - i;
        double v = L11;
        v = fma(v, f, L10); v = fma(v, f, L9); v = fma(v, f, L8); v = fma(v, f, L7); v = fma(v, f, L6); v = fma(v, f, L5);
        v = fma(v, f, L4); v = fma(v, f, L3); v = fma(v, f, L2); v = fma(v, f, L); v = fma(v, f, 1.0);
        return ldexp(v, static_cast<int>(i) + 40);
    }
    __device__ double whole(float x) const { return rint(raw(x)); }   // (sums of up to 2^13 of them are exact in fp64; a thread has at most 2^12)
    __device__ uint64_t units(float x) const { return static_cast<uint64_t>(whole(x)); }
};
__device__ inline Weights make_weights(float m, double t) { return Weights{m, 1.4426950408889634074 / t, m == INFINITY}; }

__device__ inline float log_probability(float x, const Weights& w, double t, uint64_t total)
{
    const double d = w.inf || static_cast<double>(x) == w.m ? 0.0 : (static_cast<double>(x) - w.m) / t;
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
template <typename T>
__global__ __launch_bounds__(256) void policy_short_kernel(PolicyArgs a, int64_t rows)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = blockIdx.x * 4ll + (threadIdx.x >> 6);
    if (row >= rows) return;
    const RowSettings s = row_settings(a, row);
    const float x = lane < a.n ? static_cast<float>(static_cast<const T*>(a.scores)[row * a.ld + lane]) : -INFINITY;
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

// ---- a row by one workgroup -----------------------------------------------------------------------------------------------
//
// The kept set is a prefix of the filters' order cut by min-p, so all a filter has to find is its last entry (a score with its index).
//   top-k with a small k   the k-th largest of 256 groups' maxima is a lower bound for the k-th largest score: the few entries from it on go into
//                          a list, which is sorted; everything else happens in the list.
//   otherwise              a histogram of the scores that can matter over 2048 equal parts of their range finds the part in which the count
//                          or the mass crosses; its entries go into the list.  Where they are too many (equal scores), the crossing is found digit by
//                          digit in the scores' keys.
// Every pass reads the row again, from cache: held in registers, it needs code without loops, of which the passes over 128 scores per thread took
// 300 KB.  Wavefront w has a contiguous stretch of the row, so that the draw, a search in index order, goes from wavefront to lane to entry.
constexpr int kBins = 2048, kList = 2048, kGroups = 256, kListK = 192;

struct RowShared {
    uint64_t bins[kBins];    // a histogram, or the sorted list
    uint64_t list[kList];
    uint64_t part[16], part2[16];
    uint32_t group[kGroups];
    uint32_t count;          // entries in the list
    int pick;
    uint64_t pick_sum, bound;
    double target;
};

template <typename T, int THREADS> struct Row {
    static constexpr int E = 16 / sizeof(T), WAVES = THREADS / 64;
    typedef T vec __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    const T* x;
    int n, trips, lane, wave;
    __device__ Row(const PolicyArgs& a, int64_t row)
        : x(static_cast<const T*>(a.scores) + row * a.ld), n(a.n), trips(((a.n + E - 1) / E + THREADS - 1) / THREADS), lane(threadIdx.x & 63),
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
    // f(index of the first, 16 bytes of scores) for the trips from `from` to `to`; behind the end they are -infinity
    template <typename F> __device__ __forceinline__ void each(int from, int to, const F& f) const
    {
        if (from >= to) return;
        vec next = load(from);
#pragma unroll 1
        for (int i = from; i < to; ++i) {
            const vec v = next;
            if (i + 1 < to) next = load(i + 1);
            f(first(i), v);
        }
    }
    template <typename F> __device__ __forceinline__ void each(const F& f) const { each(0, trips, f); }
    // f(score, index)
    template <typename F> __device__ __forceinline__ void each_score(const F& f) const
    {
        each([&](int at, const vec& v) {
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

// The first j of 0 .. kBins - 1 (each thread's are next to each other) at which above + f(0) + .. + f(j) reaches target, and the sum before it.  One
// does, or sh.pick stays -1.
template <int THREADS, typename F> __device__ __forceinline__ void first_reaching(RowShared& sh, const F& f, uint64_t above, double target)
{
    constexpr int PER = kBins / THREADS, WAVES = THREADS / 64;
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

// The entries of the row that `want` takes into the list, in any order; false if they do not fit.
template <typename ROW, typename F> __device__ __forceinline__ bool gather(RowShared& sh, const ROW& row, const F& want)
{
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    row.each([&](int first, const typename ROW::vec& v) {
        uint32_t hits = 0;
#pragma unroll
        for (int e = 0; e < ROW::E; ++e) hits |= first + e < row.n && want(static_cast<float>(v[e])) ? 1u << e : 0u;
        if (hits) {   // rare
            uint32_t at = atomicAdd(&sh.count, static_cast<uint32_t>(__popc(hits)));
#pragma unroll
            for (int e = 0; e < ROW::E; ++e)
                if (hits >> e & 1) {
                    if (at < kList) sh.list[at] = entry_of(static_cast<float>(v[e]), first + e);
                    ++at;
                }
        }
    });
    __syncthreads();
    return sh.count <= kList;
}

// list[0 .. count) into bins[0 .. count), descending.  Up to 256 entries each finds its place by counting
// the larger ones; more go through a bitonic network.
template <int THREADS> __device__ __forceinline__ void sort_list(RowShared& sh, int count)
{
    const int t = threadIdx.x;
    if (count <= 256) {
        if (t < count) {
            const uint64_t e = sh.list[t];
            int rank = 0;
            for (int j = 0; j < count; ++j) rank += sh.list[j] > e;
            sh.bins[rank] = e;
        }
        __syncthreads();
        return;
    }
    int size = 512;
    while (size < count) size <<= 1;
    for (int j = t; j < size; j += THREADS) sh.bins[j] = j < count ? sh.list[j] : 0;   // (no entry is 0: that is a NaN's key)
    for (int width = 2; width <= size; width <<= 1)
        for (int d = width >> 1; d; d >>= 1) {
            __syncthreads();
            for (int q = t; q < size / 2; q += THREADS) {
                const int lo = (q & ~(d - 1)) * 2 + (q & (d - 1)), hi = lo + d;
                const uint64_t x = sh.bins[lo], y = sh.bins[hi];
                if ((x < y) == ((lo & width) == 0)) { sh.bins[lo] = y; sh.bins[hi] = x; }
            }
        }
    __syncthreads();
}

// The last entry that a filter keeps, in the key's digits: by_mass the first at which the mass reaches `target`, else the first at which the count does.
// For rows whose equal scores overflow the list.
template <int THREADS, typename ROW> __device__ __forceinline__ uint64_t last_by_digits(RowShared& sh, const ROW& row, const Weights& w, bool by_mass, double target)
{
    uint32_t prefix = 0;
    uint64_t above = 0;
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bits = round == 2 ? 10 : 11;
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += THREADS) sh.bins[b] = 0;
        __syncthreads();
        row.each_score([&](float x, int index) {
            const uint32_t key = score_key(x);
            if (index >= row.n || (round > 0 && key >> (shift + bits) != prefix)) return;
            const uint64_t v = by_mass ? w.units(x) : 1;
            if (v) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.bins[(key >> shift) & ((1u << bits) - 1)]), static_cast<unsigned long long>(v));
        });
        __syncthreads();
        first_reaching<THREADS>(sh, [&](int j) { return sh.bins[kBins - 1 - j]; }, above, target);
        prefix = prefix << bits | static_cast<uint32_t>(kBins - 1 - sh.pick);
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
        row.each([&](int first, const typename ROW::vec& v8) {
            uint64_t c = 0;
#pragma unroll
            for (int e = 0; e < ROW::E; ++e) c += first + e < row.n && score_key(static_cast<float>(v8[e])) == prefix;
            const uint64_t upto = wave_scan(c);
            const int64_t before = static_cast<int64_t>(upto - c), all = static_cast<int64_t>(__shfl(upto, 63));
            if (left > 0 && left > before && left <= static_cast<int64_t>(upto)) {
                int64_t need = left - before;
#pragma unroll
                for (int e = 0; e < ROW::E; ++e)
                    if (first + e < row.n && score_key(static_cast<float>(v8[e])) == prefix && --need == 0)
                        sh.bound = entry_of(static_cast<float>(v8[e]), first + e);
            }
            left = left > all ? left - all : 0;
        });
    }
    __syncthreads();
    return sh.bound;
}

// The same through the histogram over [lo, m], into *last, which stays as it is if the crossing is not above lo.  What lies below lo is known not to matter: it
// has no mass, or lies beyond the crossing.  false if one part of the range overflows the list.
template <int THREADS, typename ROW>
__device__ __forceinline__ bool last_by_range(RowShared& sh, const ROW& row, const Weights& w, float m, float lo, bool by_mass, double target, uint64_t* last)
{
    const float per = fminf(static_cast<float>(kBins) / (m - lo), 0x1.fffffep127f);
    auto bin = [&](float x) { return min(static_cast<int>((m - x) * per), kBins - 1); };   // (rounding is monotone)
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += THREADS) sh.bins[b] = 0;
    __syncthreads();
    row.each_score([&](float x, int) {
        if (x < lo) return;
        const uint64_t v = by_mass ? w.units(x) : 1;
        atomicAdd(reinterpret_cast<unsigned long long*>(&sh.bins[bin(x)]), static_cast<unsigned long long>(v));
    });
    __syncthreads();
    uint64_t above = 0;
    int count = kBins;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {   // the part of the range, then the entry in the sorted list
        first_reaching<THREADS>(sh, [&](int j) -> uint64_t { return pass == 0 ? sh.bins[j] : j >= count ? 0 : by_mass ? w.units(entry_score(sh.bins[j])) : 1; }, above, target);
        const int b = sh.pick;
        if (b < 0) return true;
        if (pass == 1) {
            *last = sh.bins[b];
            return true;
        }
        above = sh.pick_sum;
        if (!gather(sh, row, [&](float x) { return x >= lo && bin(x) == b; })) return false;
        count = static_cast<int>(sh.count);
        sort_list<THREADS>(sh, count);
    }
    return true;
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void policy_row_kernel(PolicyArgs a)
{
    typedef Row<T, THREADS> ROW;
    constexpr int WAVES = THREADS / 64, E = ROW::E;
    __shared__ RowShared sh;
    const int64_t r = blockIdx.x;
    const int t = threadIdx.x;
    const ROW row(a, r);
    const RowSettings s = row_settings(a, r);
    // largest and smallest score, and whether there is a NaN
    float hi = -INFINITY, low = INFINITY;
    bool nan = false;
    row.each([&](int, const typename ROW::vec& v) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = static_cast<float>(v[e]);
            nan |= x != x;
            hi = fmaxf(hi, x);
            low = fminf(low, x);
        }
    });
    {   // 256 groups of threads
        float g = hi;
        if constexpr (THREADS == 1024) { g = fmaxf(g, __shfl_xor(g, 1)); g = fmaxf(g, __shfl_xor(g, 2)); }
        if (THREADS == 256 || (t & 3) == 0) sh.group[THREADS == 256 ? t : t >> 2] = score_key(g);
        for (int d = 32; d; d >>= 1) { hi = fmaxf(hi, __shfl_xor(hi, d)); low = fminf(low, __shfl_xor(low, d)); }
        if (row.lane == 0) { sh.part[row.wave] = score_key(hi); sh.part2[row.wave] = score_key(low); }
        nan = __syncthreads_or(nan);
        for (int q = 0; q < WAVES; ++q) { hi = fmaxf(hi, key_score(static_cast<uint32_t>(sh.part[q]))); low = fminf(low, key_score(static_cast<uint32_t>(sh.part2[q]))); }
    }
    const float m = hi;
    if (s.bad || nan || m == -INFINITY) {
        if (t == 0) answer(a, r, -1, not_a_number());
        return;
    }
    if (s.greedy) {
        int first = 0x7FFFFFFF;
        row.each_score([&](float x, int index) { if (x == m && index < first) first = index; });
        for (int d = 32; d; d >>= 1) first = min(first, __shfl_xor(first, d));
        __syncthreads();
        if (row.lane == 0) sh.part[row.wave] = static_cast<uint64_t>(first);
        __syncthreads();
        for (int q = 0; q < WAVES; ++q) first = min(first, static_cast<int>(sh.part[q]));
        if (t == 0) answer(a, r, first, 0.f);
        return;
    }
    const Weights w = make_weights(m, s.t);
    const double min_raw = s.min_p * kUnits;
    // ---- top-k by the list
    if (s.k && s.k <= kListK) {
        if (t < kGroups) {   // the k-th largest of the groups' maxima (the k-th of equals by number)
            const uint32_t g = sh.group[t];
            int rank = 0;
            for (int j = 0; j < kGroups; ++j) rank += sh.group[j] > g || (sh.group[j] == g && j < t);
            if (rank == s.k - 1) sh.bound = g;
        }
        __syncthreads();
        const float bound = key_score(static_cast<uint32_t>(sh.bound));
        if (gather(sh, row, [&](float x) { return x >= bound && x > -INFINITY; })) {   // (fewer than k finite scores: bound is -infinity)
            int count = static_cast<int>(sh.count);
            sort_list<THREADS>(sh, count);
            count = min(count, s.k);
            // thread j has entry j of the order
            const uint64_t e = t < count ? sh.bins[t] : 0;
            const double raw = t < count ? w.raw(entry_score(e)) : 0.0;
            const uint64_t mine = static_cast<uint64_t>(rint(raw));
            uint64_t upto = wave_scan(mine);
            __syncthreads();
            if (row.lane == 63) sh.part[row.wave] = upto;
            __syncthreads();
            uint64_t mass = 0;
            for (int q = 0; q < WAVES; ++q) { upto += q < row.wave ? sh.part[q] : 0; mass += sh.part[q]; }
            const bool keep = t < count && (t == 0 || static_cast<double>(upto - mine) < s.p * static_cast<double>(mass) || s.p >= 1.0) && raw >= min_raw;
            // back in index order: the kept ones lead the order, so entry j's place is the number of kept ones with a lower index
            const uint64_t total = block_sum<WAVES>(sh.part, keep ? mine : 0);
            if (t < kListK) sh.list[t] = keep ? e : 0;
            if (t < kListK) sh.bins[kListK + t] = keep ? mine : 0;
            __syncthreads();
            if (keep) {
                const uint64_t target = static_cast<uint64_t>(s.u * static_cast<double>(total));
                uint64_t before = 0;
                for (int j = 0; j < count; ++j) before += static_cast<uint32_t>(sh.list[j]) > static_cast<uint32_t>(e) ? sh.bins[kListK + j] : 0;   // (a lower index has a larger complement)
                if (before <= target && target < before + mine) answer(a, r, entry_index(e), log_probability(entry_score(e), w, s.t, total));
            }
            return;
        }
    }
    // ---- the last entry of the kept prefix
    uint64_t last = 0;
    // entries below m - 28.5 T round to 0 units: whether a filter keeps them shows in nothing
    const float no_mass = fmaxf(low, static_cast<float>(fmax(static_cast<double>(m) - 28.5 * s.t, -0x1.fffffep127)) - 2e-7f * fabsf(m));
    const bool flat = w.inf || !(no_mass < m) || m - no_mass == INFINITY;   // no range to divide
#pragma unroll 1
    for (int filter = 0; filter < 2; ++filter) {   // top-k by the count, then top-p by the mass of what that left
        const bool by_mass = filter == 1;
        if (by_mass ? !(s.p < 1.0) : !s.k) continue;
        double target = s.k;
        float lo = no_mass;
        if (by_mass) {
            double sum = 0.0;
            row.each([&](int first, const typename ROW::vec& v) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float x = static_cast<float>(v[e]);
                    sum += entry_of(x, first + e) >= last ? w.whole(x) : 0.0;
                }
            });
            const double mass = static_cast<double>(block_sum<WAVES>(sh.part, static_cast<uint64_t>(sum)));
            target = s.p * mass;
            // an entry is kept only if the mass from it on exceeds (1 - p) mass, and at most n entries no heavier than it make that up
            const double least = (1.0 - s.p) * mass / kUnits / (s.k ? s.k : a.n) * (1.0 - 1e-6);
            lo = fmaxf(lo, static_cast<float>(static_cast<double>(m) + s.t * log(least) * (1.0 + 1e-6)) - 1e-6f * fabsf(m));
        }
        bool by_digits = flat || !(lo < m);
        if (!by_digits) by_digits = !last_by_range<THREADS>(sh, row, w, m, lo, by_mass, target, &last);
        if (by_digits) last = last_by_digits<THREADS>(sh, row, w, by_mass, target);
    }
    // ---- the draw: per lane the kept mass of four groups of trips
    auto kept = [&](float x, int index) {
        if (x == -INFINITY || entry_of(x, index) < last) return 0.0;
        const double raw = w.raw(x);
        return raw >= min_raw ? rint(raw) : 0.0;
    };
    const int per = (row.trips + 3) / 4;
    uint64_t sums[4] = {0, 0, 0, 0};
#pragma unroll 1
    for (int g = 0; g < 4; ++g) {
        double sum = 0.0;
        row.each(g * per, min((g + 1) * per, row.trips), [&](int first, const typename ROW::vec& v) {
#pragma unroll
            for (int e = 0; e < E; ++e) sum += kept(static_cast<float>(v[e]), first + e);
        });
#pragma unroll
        for (int q = 0; q < 4; ++q) sums[q] = q == g ? static_cast<uint64_t>(sum) : sums[q];
    }
    const uint64_t mine = wave_sum(sums[0] + sums[1] + sums[2] + sums[3]);
    __syncthreads();
    if (row.lane == 0) sh.part[row.wave] = mine;
    __syncthreads();
    uint64_t total = 0;
    for (int q = 0; q < WAVES; ++q) total += sh.part[q];
    uint64_t target = static_cast<uint64_t>(s.u * static_cast<double>(total));
    int owner = -1;
    for (int q = 0; q < WAVES; ++q) {
        if (owner < 0 && target < sh.part[q]) owner = q;
        if (owner < 0) target -= sh.part[q];
    }
    if (row.wave != owner) return;
    int group = -1;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint64_t g = wave_sum(sums[q]);
        if (group < 0 && target < g) group = q;
        if (group < 0) target -= g;
    }
    bool found = false;
    row.each(group * per, min((group + 1) * per, row.trips), [&](int first, const typename ROW::vec& v) {
        if (found) return;
        double sum = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) sum += kept(static_cast<float>(v[e]), first + e);
        const uint64_t own = static_cast<uint64_t>(sum), upto = wave_scan(own), all = __shfl(upto, 63);
        if (target >= all) { target -= all; return; }
        found = true;
        if (target < upto - own || target >= upto) return;
        uint64_t at = upto - own;
        bool done = false;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = static_cast<float>(v[e]);
            at += static_cast<uint64_t>(kept(x, first + e));
            if (!done && target < at) {
                done = true;
                answer(a, r, first + e, log_probability(x, w, s.t, total));
            }
        }
    });
}

template <typename T> static void launch_policy(const PolicyArgs& a, int64_t rows, hipStream_t st)
{
    constexpr int E = 16 / sizeof(T);
    const dim3 grid(static_cast<unsigned>(rows));
    if (a.n <= 64) hipLaunchKernelGGL(policy_short_kernel<T>, dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(256), 0, st, a, rows);
    else if (a.n <= 256 * E * 8) hipLaunchKernelGGL((policy_row_kernel<T, 256>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((policy_row_kernel<T, 1024>), grid, dim3(1024), 0, st, a);
}

int enqueue_policy_sample(const PolicyArgs& a, int32_t type, int64_t rows, void* work, hipStream_t st)
{
    (void)work;
    type == DQN_TYPE_FP32 ? launch_policy<float>(a, rows, st) : type == DQN_TYPE_BF16 ? launch_policy<bf16_t>(a, rows, st) : launch_policy<_Float16>(a, rows, st);
    DQN_LAUNCH_CHECK();
    return DQN_OK;
}

}  // namespace dqn

using namespace dqn;

extern "C" {

size_t policy_sample_workspace(int64_t rows, int64_t n)
{
    (void)rows; (void)n;
    return 0;
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
    if (int rc = check_stream_device(who, stream)) return rc;
    const PolicyArgs a{scores, ld, static_cast<int32_t>(n), temperature, top_k, top_p, min_p, u, 0, 0, index, logp};
    return enqueue_policy_sample(a, type, rows, work, static_cast<hipStream_t>(stream));
}

}  // extern "C"
