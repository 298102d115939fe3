// Drawing an index from a row of scores under temperature, top-k, top-p and min-p (include/dqn_mi355.h: policy_sample).
#include "policy.h"

#include "gemm_mfma.h"

namespace dqn {

// ---- weights ------------------------------------------------------------------------------------------------------------
//
// w = exp((x - m) / T) in fp64 and, for every sum, as a whole multiple of 2^-40: integer sums are the same in any order (histograms are
// filled by atomics, rows are split), and with n <= 2^22 they fit 63 bits.
constexpr double kPolicyUnit = 0x1p40;

struct RowSettings {
    double inv_t, p, min_p, u;
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
    s.inv_t = 1.0 / static_cast<double>(t);
    s.p = p; s.min_p = fmin(static_cast<double>(mp), 1.0);
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

__device__ inline double weight(float x, float m, double inv_t) { return x == m ? 1.0 : exp((static_cast<double>(x) - static_cast<double>(m)) * inv_t); }
__device__ inline uint64_t fixed(double w) { return static_cast<uint64_t>(w * kPolicyUnit + 0.5); }

// ---- a row by one workgroup -----------------------------------------------------------------------------------------------
//
// The kept set is a prefix of the order (score descending, index ascending) cut by min-p, so all a filter has to find is its last entry: a
// score and, among equal scores, how many of them.  That is found like a digit-wise selection: a histogram over the leading 11 bits of the
// keys (entries and mass per bin), the bin in which the count or the mass crosses its target, then the same inside that bin for the next
// 11 and the last 10 bits.  The draw itself is a search for the crossing of a prefix sum in index order: the wavefronts sum one
// part of the range each, then the part that holds the crossing is divided again.
constexpr int kRowThreads = 512, kRowWaves = kRowThreads / 64, kBins = 2048;

struct RowShared {
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint64_t part[kRowWaves];
    uint64_t part2[kRowWaves];
    uint32_t pick_bin; uint64_t pick_count, pick_mass;
};

template <typename T> struct Row {
    const T* x; int n; float m; double inv_t;
    __device__ float at(int i) const { return static_cast<float>(x[i]); }
    __device__ uint64_t fixed_at(float v) const { return fixed(weight(v, m, inv_t)); }
};

__device__ inline uint64_t wave_sum(uint64_t v)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Lowest i of [0, n) at which the sum of f over 0..i exceeds `target` -- or, with a share u instead, u * (the whole sum), which is returned in *total.
// n (which there is always such an i below) if the whole sum does not exceed it.
template <typename F> __device__ inline int locate(RowShared& sh, int n, const F& f, uint64_t target, double u, bool by_share, uint64_t* total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int lo = 0, len = n;
    bool first = true;
    while (true) {
        const int sub = ((len + kRowWaves - 1) / kRowWaves + 63) / 64 * 64;
        uint64_t mine = 0;
        const int a = lo + wave * sub, b = min(lo + len, a + sub);
        for (int i = a + lane; i < b; i += 64) mine += f(i);
        mine = wave_sum(mine);
        __syncthreads();
        if (lane == 0) sh.part[wave] = mine;
        __syncthreads();
        uint64_t before = 0;
        if (first && by_share) {
            uint64_t all = 0;
            for (int q = 0; q < kRowWaves; ++q) all += sh.part[q];
            *total = all;
            target = static_cast<uint64_t>(u * static_cast<double>(all));
        }
        first = false;
        int pick = -1;
        for (int q = 0; q < kRowWaves; ++q) {
            if (pick < 0 && before + sh.part[q] > target) pick = q;
            if (pick < 0) before += sh.part[q];
        }
        if (pick < 0) return n;
        target -= before;
        const int end = lo + len;
        lo += pick * sub;
        len = min(sub, end - lo);
        if (sub == 64) break;
    }
    uint64_t v = lane < len ? f(lo + lane) : 0;   // every wavefront the same
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    const uint64_t hit = __ballot(v > target);
    return hit ? lo + __builtin_ctzll(hit) : n;
}

// The last entry that a filter keeps: its key, how many entries of that key (in index order), and the mass up to it.
struct Last { uint32_t key; uint32_t ties, all_ties; uint64_t mass; };

// by_mass: the first entry (in order) at which the mass reaches `target`; else the first at which the count reaches it.
template <typename T> __device__ inline Last select_last(RowShared& sh, const Row<T>& row, bool by_mass, double target)
{
    uint32_t prefix = 0;
    uint64_t above_count = 0, above_mass = 0;
    const int shifts[3] = {21, 10, 0};
    uint32_t in_bin = 0;
    for (int round = 0; round < 3; ++round) {
        const int shift = shifts[round], bits = round == 2 ? 10 : 11;
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += kRowThreads) { sh.count[b] = 0; sh.mass[b] = 0; }
        __syncthreads();
        for (int i = threadIdx.x; i < row.n; i += kRowThreads) {
            const float v = row.at(i);
            const uint32_t key = score_key(v);
            if (round > 0 && (key >> (shift + bits)) != prefix) continue;
            const uint32_t b = (key >> shift) & ((1u << bits) - 1);
            atomicAdd(&sh.count[b], 1u);
            const uint64_t w = row.fixed_at(v);
            if (w) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]), static_cast<unsigned long long>(w));
        }
        __syncthreads();
        // bins from the top down: thread t has four of them
        uint32_t c[4]; uint64_t w[4];
        uint64_t cs = 0, ws = 0;
        for (int j = 0; j < 4; ++j) {
            const int b = kBins - 1 - (static_cast<int>(threadIdx.x) * 4 + j);
            c[j] = sh.count[b]; w[j] = sh.mass[b];
            cs += c[j]; ws += w[j];
        }
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        uint64_t ci = cs, wi = ws;
        for (int d = 1; d < 64; d <<= 1) {
            const uint64_t co = __shfl_up(ci, d), wo = __shfl_up(wi, d);
            if (lane >= d) { ci += co; wi += wo; }
        }
        __syncthreads();
        if (lane == 63) { sh.part[wave] = ci; sh.part2[wave] = wi; }
        __syncthreads();
        uint64_t c0 = above_count + ci - cs, w0 = above_mass + wi - ws;
        for (int q = 0; q < wave; ++q) { c0 += sh.part[q]; w0 += sh.part2[q]; }
        for (int j = 0; j < 4; ++j) {   // exactly one bin crosses
            const bool was = (by_mass ? static_cast<double>(w0) : static_cast<double>(c0)) >= target;
            const bool is = (by_mass ? static_cast<double>(w0 + w[j]) : static_cast<double>(c0 + c[j])) >= target;
            if (!was && is) { sh.pick_bin = kBins - 1 - (threadIdx.x * 4 + j); sh.pick_count = c0; sh.pick_mass = w0; }
            c0 += c[j]; w0 += w[j];
        }
        __syncthreads();
        const uint32_t bin = sh.pick_bin;
        above_count = sh.pick_count; above_mass = sh.pick_mass;
        in_bin = sh.count[bin];
        prefix = prefix << bits | bin;
    }
    Last last;
    last.key = prefix;
    last.all_ties = in_bin;
    const uint64_t w = row.fixed_at(key_score(prefix));
    uint64_t r;
    if (by_mass) {
        r = w ? static_cast<uint64_t>((target - static_cast<double>(above_mass)) / static_cast<double>(w)) : 1;
        r = r < 1 ? 1 : r > in_bin ? in_bin : r;
        while (r > 1 && static_cast<double>(above_mass + (r - 1) * w) >= target) --r;
        while (r < in_bin && static_cast<double>(above_mass + r * w) < target) ++r;
    } else {
        r = static_cast<uint64_t>(target) - above_count;
    }
    last.ties = static_cast<uint32_t>(r);
    last.mass = above_mass + r * w;
    return last;
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void policy_row_kernel(PolicyArgs a)
{
    __shared__ RowShared sh;
    const int64_t r = blockIdx.x;
    const RowSettings s = row_settings(a, r);
    Row<T> row{static_cast<const T*>(a.scores) + r * a.ld, a.n, 0.f, s.inv_t};
    // the maximum with its lowest index, and whether there is a NaN
    uint64_t best = 0;
    bool nan = false;
    for (int i = threadIdx.x; i < a.n; i += kRowThreads) {
        const float v = row.at(i);
        nan |= v != v;
        const uint64_t c = static_cast<uint64_t>(score_key(v)) << 32 | static_cast<uint32_t>(~i);
        best = c > best ? c : best;
    }
    for (int d = 32; d; d >>= 1) {
        const uint64_t o = __shfl_xor(best, d);
        best = o > best ? o : best;
    }
    if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = best;
    nan = __syncthreads_or(nan);
    for (int q = 0; q < kRowWaves; ++q) best = sh.part[q] > best ? sh.part[q] : best;
    const float m = key_score(static_cast<uint32_t>(best >> 32));
    auto answer = [&](int32_t index, float logp) {
        if (threadIdx.x == 0) {
            a.index[r] = index;
            if (a.logp) a.logp[r] = logp;
        }
    };
    if (s.bad || nan || a.n == 0 || m == -INFINITY) return answer(-1, __uint_as_float(0x7FC00000u));
    if (s.greedy) return answer(static_cast<int32_t>(~static_cast<uint32_t>(best)), 0.f);
    row.m = m;
    Last last{0, 0xFFFFFFFFu, 0xFFFFFFFFu, 0};
    bool cut = false;
    double mass = 0.0;
    if (s.k) {
        last = select_last(sh, row, false, static_cast<double>(s.k));
        cut = true;
        mass = static_cast<double>(last.mass);
    }
    if (s.p < 1.0) {
        if (!s.k) {
            uint64_t all = 0;
            locate(sh, a.n, [&](int i) { return row.fixed_at(row.at(i)); }, 0, 0.0, true, &all);
            mass = static_cast<double>(all);
        }
        last = select_last(sh, row, true, s.p * mass);
        cut = true;
    }
    int last_index = a.n;   // the last entry kept among those of last.key
    uint64_t ignored = 0;
    if (cut && last.ties < last.all_ties)
        last_index = locate(sh, a.n, [&](int i) { return static_cast<uint64_t>(score_key(row.at(i)) == last.key); }, last.ties - 1, 0.0, false, &ignored);
    uint64_t total = 0;
    const int pick = locate(sh, a.n, [&](int i) -> uint64_t {
        const float v = row.at(i);
        const uint32_t key = score_key(v);
        if (key < last.key || (key == last.key && i > last_index)) return 0;
        const double w = weight(v, m, s.inv_t);
        return w >= s.min_p ? fixed(w) : 0;
    }, 0, s.u, true, &total);
    const float v = row.at(pick);
    const double d = v == m ? 0.0 : (static_cast<double>(v) - static_cast<double>(m)) * s.inv_t;
    answer(pick, static_cast<float>(d - log(static_cast<double>(total) / kPolicyUnit)));
}

int enqueue_policy_sample(const PolicyArgs& a, int32_t type, int64_t rows, void* work, hipStream_t st)
{
    (void)work;
    auto kern = type == DQN_TYPE_FP32 ? policy_row_kernel<float> : type == DQN_TYPE_BF16 ? policy_row_kernel<bf16_t> : policy_row_kernel<_Float16>;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(rows)), dim3(kRowThreads), 0, st, a);
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
