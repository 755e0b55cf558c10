// Draws from a truncated temperature softmax, with settings for each row (tkv_filter_sample).
//
// Tokens are ordered by (logit descending, index ascending), here as one 53-bit number a token: the logit's bits,
// mapped so that larger means larger, above the complement of the index.  All numbers of a row differ, and what
// top-k, top-p and min-p keep is everything from a threshold up, so truncation is finding that threshold:
//   top-k   the k-th number from above;
//   top-p   the number at which the sum of the weights from above reaches top_p times the (top-k) total;
//   min-p   a bound on the weight itself.
// The first two are found by histograms over the numbers: 2,048 bins of the interval that still holds the threshold,
// with each bin's count and weight, until that interval holds few enough tokens to sort.
//
// Weights are computed in fp64, w = 2^((l - max) log2(e) / T).  Histogram sums are integers, w in units of 2^-42, so
// that they do not depend on the order of the atomics; they decide where top-p ends to 2^-43 of the largest weight a
// token.  The draws' sums are fp64 in a fixed order.
#include <hip/hip_runtime.h>
#include <cstdint>

#include "internal.h"

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kList = 2048;           // tokens that are sorted
constexpr int kIdxBits = 21;          // vocabularies of up to 2^21 tokens
constexpr int kPerLane = 16;          // contiguous tokens of a lane where draws are summed
constexpr int kTile = 64 * kPerLane;
constexpr int kMaxTiles = (1 << kIdxBits) / kTile;
constexpr int kMaxPotential = 1024;
constexpr double kUnit = 4398046511104.0;  // 2^42

typedef float f32x4_t __attribute__((ext_vector_type(4), aligned(4)));        // rows may start at any element
typedef uint16_t u16x8_t __attribute__((ext_vector_type(8), aligned(2)));

struct Args {
    int32_t n_rows, vocab;
    const void* logits;
    int64_t stride;
    const float *temperature, *top_p, *min_p;
    const int32_t* top_k;
    const float* uniform;
    const int32_t* draw_off;
    int32_t n_draws;
    int32_t *token, *count, *n_groups;
};

// Larger logits have larger keys; -0 and 0 have one.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ uint64_t number_of(float x, int i) {
    return static_cast<uint64_t>(key_of(x)) << kIdxBits | static_cast<uint64_t>((1 << kIdxBits) - 1 - i);
}
__device__ __forceinline__ float bf16_f32(uint16_t u) { return __uint_as_float(static_cast<uint32_t>(u) << 16); }

template <bool BF16>
struct Logits {
    const void* p;
    int vocab;
    __device__ __forceinline__ float at(int i) const {
        return BF16 ? bf16_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
    }
    // f(index, logit) for every logit, shared out over the workgroup
    template <class F>
    __device__ __forceinline__ void each(F f) const {
        constexpr int V = BF16 ? 8 : 4;
        const int whole = vocab / V;
        for (int i = threadIdx.x; i < whole; i += kThreads) {
            if constexpr (BF16) {
                const u16x8_t x = reinterpret_cast<const u16x8_t*>(p)[i];
#pragma unroll
                for (int e = 0; e < V; ++e) f(V * i + e, bf16_f32(x[e]));
            } else {
                const f32x4_t x = reinterpret_cast<const f32x4_t*>(p)[i];
#pragma unroll
                for (int e = 0; e < V; ++e) f(V * i + e, x[e]);
            }
        }
        for (int i = V * whole + threadIdx.x; i < vocab; i += kThreads) f(i, at(i));
    }
    // this lane's 16 of the tile that starts at a0 (-inf past the row)
    __device__ __forceinline__ void lane16(int a0, int lane, float (&x)[kPerLane]) const {
        const int a = a0 + lane * kPerLane;
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) x[e] = a + e < vocab ? at(a + e) : -INFINITY;
    }
};

__device__ __forceinline__ double shfl_up_d(double v, int o) { return __shfl_up(v, o); }

// Inclusive scan over a wave, in a fixed pattern.
template <class T>
__device__ __forceinline__ T wave_scan(T v, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T u = __shfl_up(v, o);
        if (lane >= o) v += u;
    }
    return v;
}

// Exclusive scan over the workgroup and the total; `part` holds a value a wave.
template <class T>
__device__ __forceinline__ T block_scan(T v, T* part, T& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const T incl = wave_scan(v, lane);
    __syncthreads();  // part is free
    if (lane == 63) part[w] = incl;
    __syncthreads();
    T before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i == w) before = total;
        total += part[i];
    }
    return before + incl - v;
}

// Bitonic sort of n (a power of two) numbers, descending.
template <class T>
__device__ __forceinline__ void sort_down(T* a, int n) {
    for (int k = 2; k <= n; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            __syncthreads();
            for (int t = threadIdx.x; t < n / 2; t += kThreads) {
                const int i = 2 * j * (t / j) + t % j, p = i + j;
                const T x = a[i], y = a[p];
                if ((x < y) == ((i & k) == 0)) a[i] = y, a[p] = x;
            }
        }
    __syncthreads();
}
__device__ __forceinline__ int pow2_at_least(int n) { return n <= 1 ? 1 : 1 << (32 - __builtin_clz(n - 1)); }

struct Shared {
    union {
        struct {
            uint64_t mass[kBins];
            uint32_t cnt[kBins];
        } h;
        uint64_t list[kList];
        double tile[kMaxTiles + 1];  // the draws' tile prefixes
    };
    uint64_t part[kWaves];
    double partd[kWaves];
    union {
        uint32_t draw[kMaxPotential];  // complements of the tokens drawn
        float red[2 * kWaves];
    };
    int32_t start[kMaxPotential + 1];
    uint64_t u0, u1;
    double d0;
    int i0, i1;
};

// The distribution of a row.
template <bool BF16>
struct Row {
    Logits<BF16> x;
    double top, c;  // w = 2^((x - top) c)
    __device__ __forceinline__ double weight(float v) const { return exp2((static_cast<double>(v) - top) * c); }
    __device__ __forceinline__ uint64_t units(float v) const { return static_cast<uint64_t>(weight(v) * kUnit + 0.5); }
};

// Where a run from above, of numbers in [lo, hi], reaches a target: its last number, and the run's weight.
struct Cut {
    uint64_t number, mass;
};

// BY_MASS: the target is `share` of the whole weight at or above lo (all of it in the first histogram), else a count.
template <bool BF16, bool BY_MASS>
__device__ Cut find_cut(Shared& s, const Row<BF16>& row, uint64_t lo, uint64_t hi, uint64_t target, double share) {
    const int t = threadIdx.x;
    uint64_t above_c = 0, above_m = 0;
    double want = static_cast<double>(target);
    const uint64_t floor = lo;
    for (bool first = true;; first = false) {
        const int bits = 64 - __builtin_clzll(hi - lo | 1), shift = bits > 11 ? bits - 11 : 0;
        __syncthreads();
        for (int i = t; i < kBins; i += kThreads) s.h.mass[i] = 0, s.h.cnt[i] = 0;
        __syncthreads();
        row.x.each([&](int i, float v) {
            const uint64_t n = number_of(v, i);
            if (n < lo || n > hi) return;
            const int b = static_cast<int>((n - lo) >> shift);
            atomicAdd(&s.h.cnt[b], 1u);
            atomicAdd(reinterpret_cast<unsigned long long*>(&s.h.mass[b]), static_cast<unsigned long long>(row.units(v)));
        });
        __syncthreads();
        // thread t takes bins from the top down: kBins - 1 - per t and the next below
        constexpr int per = kBins / kThreads;
        uint64_t c[per], m[per], cs = 0, ms = 0, total_c, total_m;
#pragma unroll
        for (int e = 0; e < per; ++e) {
            const int b = kBins - 1 - (per * t + e);
            cs += c[e] = s.h.cnt[b];
            ms += m[e] = s.h.mass[b];
        }
        uint64_t before_c = above_c + block_scan(cs, s.part, total_c);
        uint64_t before_m = above_m + block_scan(ms, s.part, total_m);
        if (BY_MASS && first) want = share * static_cast<double>(total_m);
        if (t == 0) s.i0 = -1;
        __syncthreads();
        uint64_t bc = before_c, bm = before_m;
#pragma unroll
        for (int e = 0; e < per; ++e) {
            const uint64_t ac = bc + c[e], am = bm + m[e];
            const bool reached = BY_MASS ? static_cast<double>(am) >= want : ac >= target;
            const bool was = BY_MASS ? static_cast<double>(bm) >= want : bc >= target;
            // (the first bin that holds anything, if nothing is wanted)
            if (c[e] > 0 && reached && (!was || bc == 0)) {
                s.i0 = kBins - 1 - (per * t + e);
                s.i1 = static_cast<int>(c[e]);
                s.u0 = bc, s.u1 = bm;
            }
            bc = ac, bm = am;
        }
        __syncthreads();
        if (s.i0 < 0) return Cut{floor, above_m + total_m};  // all of it is less than the target
        const int bin = s.i0, n = s.i1;
        above_c = s.u0, above_m = s.u1;
        lo += static_cast<uint64_t>(bin) << shift;
        hi = lo + ((uint64_t{1} << shift) - 1);
        if (n > kList) continue;
        // few enough to sort
        __syncthreads();
        if (t == 0) s.i0 = 0;
        __syncthreads();
        row.x.each([&](int i, float v) {
            const uint64_t x = number_of(v, i);
            if (x >= lo && x <= hi) s.list[atomicAdd(&s.i0, 1)] = x;
        });
        const int size = pow2_at_least(n);
        for (int i = n + t; i < size; i += kThreads) s.list[i] = 0;
        sort_down(s.list, size);
        constexpr int many = kList / kThreads;
        uint64_t mine = 0, total, w[many];
#pragma unroll
        for (int e = 0; e < many; ++e) {
            const int i = many * t + e;
            w[e] = 0;
            if (i < n) {
                const int idx = (1 << kIdxBits) - 1 - static_cast<int>(s.list[i] & ((1 << kIdxBits) - 1));
                w[e] = row.units(row.x.at(idx));
            }
            mine += w[e];
        }
        uint64_t run = above_m + block_scan(mine, s.part, total);
        if (t == 0) s.u0 = s.list[n - 1], s.u1 = above_m + total;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < many; ++e) {
            const int i = many * t + e;
            const uint64_t next = run + w[e];
            const bool reached = BY_MASS ? static_cast<double>(next) >= want : above_c + i + 1 >= target;
            const bool was = BY_MASS ? static_cast<double>(run) >= want : above_c + i >= target;
            if (i < n && reached && (!was || above_c + i == 0)) s.u0 = s.list[i], s.u1 = next;
            run = next;
        }
        __syncthreads();
        const Cut cut{s.u0, s.u1};
        __syncthreads();
        return cut;
    }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void filter_sample(Args a) {
    __shared__ Shared s;
    const int r = blockIdx.x, t = threadIdx.x, lane = t & 63;
    const int w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int off = a.draw_off[r], n = a.draw_off[r + 1] - off;
    // (offsets are device data: a row outside the arrays reads and writes nothing)
    if (off < 0 || off > a.n_draws || n < 0 || n > a.n_draws - off || n > kMaxPotential) {
        if (t == 0) a.n_groups[r] = -1;
        return;
    }
    for (int i = t; i < n; i += kThreads) a.token[off + i] = -1, a.count[off + i] = 0;
    const float temp = a.temperature[r], p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
    int k = a.top_k ? a.top_k[r] : 0;
    const bool valid = temp >= 0.f && temp < INFINITY && p >= 0.f && p <= 1.f && min_p >= 0.f && min_p <= 1.f && k >= 0;
    if (!valid || n == 0) {
        if (t == 0) a.n_groups[r] = valid ? 0 : -1;
        return;
    }
    if (temp == 0.f) k = 1;
    if (k == 0 || k > a.vocab) k = a.vocab;
    Row<BF16> row{{static_cast<const char*>(a.logits) + r * a.stride * (BF16 ? 2 : 4), a.vocab}, 0., 1.};

    // the largest and smallest finite logits
    float top = -INFINITY, low = INFINITY;
    bool nan = false;
    row.x.each([&](int, float v) {
        nan |= v != v;
        top = fmaxf(top, v);
        low = fminf(low, v == -INFINITY ? INFINITY : v);
    });
    if (nan) top = INFINITY;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o)), low = fminf(low, __shfl_xor(low, o));
    if (lane == 0) s.red[w] = top, s.red[kWaves + w] = low;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = fmaxf(top, s.red[i]), low = fminf(low, s.red[kWaves + i]);
    if (top == INFINITY || top == -INFINITY) {
        if (t == 0) a.n_groups[r] = -1;
        return;
    }
    __syncthreads();
    row.top = top;
    row.c = temp == 0.f ? 1. : 1.4426950408889634 / static_cast<double>(temp);

    const uint64_t lo = static_cast<uint64_t>(key_of(low)) << kIdxBits;
    const uint64_t hi = number_of(top, 0);
    uint64_t cut = 0;
    if (k < a.vocab) {
        const Cut c = find_cut<BF16, false>(s, row, lo, hi, static_cast<uint64_t>(k), 0.);
        cut = c.number;
    }
    if (p < 1.f) cut = find_cut<BF16, true>(s, row, cut > lo ? cut : lo, hi, 0, static_cast<double>(p)).number;
    const double bound = static_cast<double>(min_p);
    auto kept = [&](int i, float v) {
        const double x = row.weight(v);
        return number_of(v, i) >= cut && x >= bound ? x : 0.;
    };

    // the kept weight of each tile, in token order within a lane
    const int tiles = (a.vocab + kTile - 1) / kTile;
    auto lane_sum = [&](const float (&x)[kPerLane], int first) {
        double sum = 0.;
#pragma unroll
        for (int e = 0; e < kPerLane; ++e)
            if (first + e < a.vocab) sum += kept(first + e, x[e]);
        return sum;
    };
    for (int i = w; i < tiles; i += kWaves) {
        float x[kPerLane];
        row.x.lane16(i * kTile, lane, x);
        const double sum = wave_scan(lane_sum(x, i * kTile + lane * kPerLane), lane);
        if (lane == 63) s.tile[i + 1] = sum;
    }
    __syncthreads();
    if (w == 0) {
        double run = 0.;
        for (int i0 = 0; i0 < tiles; i0 += 64) {
            const double incl = run + wave_scan(i0 + lane < tiles ? s.tile[i0 + lane + 1] : 0., lane);
            if (i0 + lane < tiles) s.tile[i0 + lane + 1] = incl;
            run = __shfl(incl, 63);
        }
        if (lane == 0) s.tile[0] = 0.;
    }
    __syncthreads();
    const double total = s.tile[tiles];

    // one wave a draw: its tile, the lane in it, the token
    for (int d = w; d < n; d += kWaves) {
        const double target = static_cast<double>(a.uniform[off + d]) * total;
        int b = 0, e = tiles;  // the first tile that ends past the target
        while (b < e) {
            const int mid = (b + e) >> 1;
            if (s.tile[mid + 1] > target) e = mid; else b = mid + 1;
        }
        if (b == tiles) {  // none: the last with a weight
            b = tiles - 1;
            while (b > 0 && !(s.tile[b + 1] > s.tile[b])) --b;
        }
        b = __builtin_amdgcn_readfirstlane(b);
        float x[kPerLane];
        const int first = b * kTile + lane * kPerLane;
        row.x.lane16(b * kTile, lane, x);
        const double sum = lane_sum(x, first);
        const double incl = s.tile[b] + wave_scan(sum, lane);
        const uint64_t has = __builtin_amdgcn_ballot_w64(sum > 0.);
        const uint64_t past = has & __builtin_amdgcn_ballot_w64(incl > target);
        const int who = past ? __builtin_ctzll(past) : has ? 63 - __builtin_clzll(has) : 0;
        if (lane == who) {
            double acc = incl - sum;
            int pick = -1, last = 0;
#pragma unroll
            for (int q = 0; q < kPerLane; ++q) {
                const double y = first + q < a.vocab ? kept(first + q, x[q]) : 0.;
                acc += y;
                if (y > 0.) {
                    last = first + q;
                    if (pick < 0 && acc > target) pick = last;
                }
            }
            s.draw[d] = ~static_cast<uint32_t>(pick >= 0 ? pick : last);
        }
    }
    __syncthreads();

    // group by token: sorted, then the start of each run
    const int size = pow2_at_least(n);
    for (int i = n + t; i < size; i += kThreads) s.draw[i] = 0;
    sort_down(s.draw, size);
    constexpr int per = kMaxPotential / kThreads;
    uint64_t firsts = 0, groups;
    bool is[per];
#pragma unroll
    for (int e = 0; e < per; ++e) {
        const int i = per * t + e;
        is[e] = i < n && (i == 0 || s.draw[i] != s.draw[i - 1]);
        firsts += is[e];
    }
    uint64_t at = block_scan(firsts, s.part, groups);
#pragma unroll
    for (int e = 0; e < per; ++e)
        if (is[e]) s.start[at++] = per * t + e;
    if (t == 0) s.start[groups] = n;
    __syncthreads();
    for (int i = t; i < static_cast<int>(groups); i += kThreads) {
        a.token[off + i] = static_cast<int32_t>(~s.draw[s.start[i]]);
        a.count[off + i] = s.start[i + 1] - s.start[i];
    }
    if (t == 0) a.n_groups[r] = static_cast<int32_t>(groups);
}

}  // namespace

int tkv::launch_filter_sample(const FilterCall& f, void* stream) {
    Args a{};
    a.n_rows = f.n_rows, a.vocab = f.vocab, a.logits = f.logits, a.stride = f.stride;
    a.temperature = f.temperature, a.top_k = f.top_k, a.top_p = f.top_p, a.min_p = f.min_p;
    a.uniform = f.uniform, a.draw_off = f.draw_off, a.n_draws = f.n_draws;
    a.token = f.token, a.count = f.count, a.n_groups = f.n_groups;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (f.logit_type == TKV_LOGITS_BF16)
        filter_sample<true><<<dim3(static_cast<unsigned>(f.n_rows)), dim3(kThreads), 0, st>>>(a);
    else
        filter_sample<false><<<dim3(static_cast<unsigned>(f.n_rows)), dim3(kThreads), 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TKV_OK : set_error(TKV_EHIP, "tkv_filter_sample launch: %s", hipGetErrorString(e));
}
