// Draws from a truncated temperature softmax, with settings for each row (tkv_filter_sample).
//
// Tokens are ordered by (logit descending, index ascending), here as one 53-bit number a token: the logit's bits,
// mapped so that larger means larger, above the complement of the index.  All numbers of a row differ, and what
// top-k, top-p and min-p keep is everything from a threshold up, so truncation is finding that threshold:
//   top-k   the k-th number from above;
//   top-p   the number at which the sum of the weights from above reaches top_p times the (top-k) total;
//   min-p   a bound on the weight itself.
//
// Two kernels.  filter_scan streams the logits once, a wave per 2,048: the largest logit of every run of 32, and, for
// rows whose whole weight is asked for (top-p without top-k, or no truncation), the tile's weight relative to its
// largest.  filter_draw then takes a workgroup a row.  The runs' maxima bound the threshold from below (the k-th
// largest of them is at most the k-th largest logit), so only the few runs above that bound are read again, their
// tokens above it sorted, cut and drawn from.  A row whose threshold lies deeper than kList tokens is read again
// whole: histograms over the numbers, 2,048 bins of the interval that still holds the threshold, with each bin's count
// and weight, until that interval holds few enough tokens to sort.
//
// Weights are computed in fp64, w = 2^((l - max) log2(e) / T), and summed in a fixed order.  Histogram sums are
// integers, w in units of 2^-42, so that they do not depend on the order of the atomics; they decide where top-p ends
// to 2^-43 of the largest weight a token.
#include <hip/hip_runtime.h>
#include <cstdint>

#include "internal.h"

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kList = 2048;           // tokens that are sorted
constexpr int kIdxBits = 21;          // vocabularies of up to 2^21 tokens
constexpr int kRun = 32;              // tokens of a lane in a tile
constexpr int kTile = tkv::kFilterTile;
static_assert(kTile == 64 * kRun, "a run a lane");
constexpr int kScanThreads = 256;
constexpr int kSparseK = 1024;        // largest top-k that is looked for among the runs' maxima
constexpr int kSparseP = 256;         // runs looked into for top-p
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
    int32_t tiles;      // a row's
    float* run_max;     // [n_rows][tiles][64]
    double* tile_sum;   // [n_rows][tiles]: weight relative to the tile's largest
};

// A row's settings and draws.
struct Settings {
    float temp, p, min_p;
    int k;        // vocab: all
    int off, n;
    bool inside;  // its draws are inside the arrays
    bool valid;
    // the weight of all of the row's tokens decides something
    __device__ __forceinline__ bool whole(int vocab) const { return k >= vocab && (p < 1.f || min_p <= 0.f); }
    __device__ __forceinline__ double scale() const { return temp == 0.f ? 1. : 1.4426950408889634 / static_cast<double>(temp); }
};
__device__ __forceinline__ Settings settings_of(const Args& a, int r) {
    Settings s;
    s.off = a.draw_off[r];
    const int end = a.draw_off[r + 1];
    s.inside = s.off >= 0 && s.off <= a.n_draws && end >= s.off && end <= a.n_draws && end - s.off <= kMaxPotential;
    s.n = s.inside ? end - s.off : 0;
    s.temp = a.temperature[r];
    s.p = a.top_p ? a.top_p[r] : 1.f;
    s.min_p = a.min_p ? a.min_p[r] : 0.f;
    s.k = a.top_k ? a.top_k[r] : 0;
    s.valid = s.temp >= 0.f && s.temp < INFINITY && s.p >= 0.f && s.p <= 1.f && s.min_p >= 0.f && s.min_p <= 1.f && s.k >= 0;
    if (s.temp == 0.f) s.k = 1;
    if (s.k == 0 || s.k > a.vocab) s.k = a.vocab;
    return s;
}

// 2^t for t <= 0, to 2^-52: t's nearest integer by adding 1.5 * 2^52, and the series of exp on [-ln 2 / 2, ln 2 / 2],
// whose first omitted term is below 2^-52.
__device__ __forceinline__ double exp2_neg(double t) {
    constexpr double kRound = 6755399441055744.0;
    t = fmax(t, -1100.);
    const double r = t + kRound;
    const int n = static_cast<int>(__double_as_longlong(r));
    const double f = (t - (r - kRound)) * 0.6931471805599453;
    double y = 1. / 479001600.;
    y = fma(y, f, 1. / 39916800.);
    y = fma(y, f, 1. / 3628800.);
    y = fma(y, f, 1. / 362880.);
    y = fma(y, f, 1. / 40320.);
    y = fma(y, f, 1. / 5040.);
    y = fma(y, f, 1. / 720.);
    y = fma(y, f, 1. / 120.);
    y = fma(y, f, 1. / 24.);
    y = fma(y, f, 1. / 6.);
    y = fma(y, f, .5);
    y = fma(y, f, 1.);
    y = fma(y, f, 1.);
    return ldexp(y, n);
}

// Larger logits have larger keys; -0 and 0 have one.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ uint64_t number_of(float x, int i) {
    return static_cast<uint64_t>(key_of(x)) << kIdxBits | static_cast<uint64_t>((1 << kIdxBits) - 1 - i);
}
// The logit of a number (0 for -0).
__device__ __forceinline__ float logit_of(uint64_t n) {
    const uint32_t k = static_cast<uint32_t>(n >> kIdxBits);
    return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu));
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
    // this lane's run of the tile that starts at a0: kPieces pieces of V tokens, 64 V apart (-inf past the row)
    static constexpr int V = BF16 ? 8 : 4, kPieces = kRun / V;
    static __device__ __forceinline__ int token(int a0, int lane, int piece) { return a0 + (piece * 64 + lane) * V; }
    __device__ __forceinline__ void piece(int a, float (&x)[V]) const {
        if (a + V <= vocab) {
            if constexpr (BF16) {
                const u16x8_t y = *reinterpret_cast<const u16x8_t*>(static_cast<const uint16_t*>(p) + a);
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = bf16_f32(y[e]);
            } else {
                const f32x4_t y = *reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p) + a);
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = y[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = a + e < vocab ? at(a + e) : -INFINITY;
        }
    }
    // kRun consecutive tokens of a tile for each lane
    __device__ __forceinline__ void consecutive(int a0, int lane, float (&x)[kPieces][V]) const {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) piece(a0 + lane * kRun + j * V, x[j]);
    }
    __device__ __forceinline__ void run(int a0, int lane, float (&x)[kPieces][V]) const {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) piece(token(a0, lane, j), x[j]);
    }
};

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
        struct {
            uint64_t list[kList];  // the tokens above the bound
            union {
                struct {
                    uint32_t hist[kBins / 2];
                    int32_t runs[kList];
                };
                double cdf[kList];
            };
            int32_t hits[kList];  // draws of each kept token
        };
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
    int i0, i1, i2;
};

// The distribution of a row.
template <bool BF16>
struct Row {
    Logits<BF16> x;
    double top, c;  // w = 2^((x - top) c)
    __device__ __forceinline__ double weight(float v) const { return exp2_neg((static_cast<double>(v) - top) * c); }
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

// A wave a tile: the runs' maxima (+inf where a logit is NaN), and the tile's weight where the row asks for it.
template <bool BF16>
__global__ __launch_bounds__(kScanThreads) void filter_scan(Args a) {
    const int lane = threadIdx.x & 63;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * (kScanThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = static_cast<int>(id / a.tiles), tile = static_cast<int>(id - static_cast<int64_t>(r) * a.tiles);
    if (r >= a.n_rows) return;
    const Settings s = settings_of(a, r);
    if (!s.inside || !s.valid || s.n == 0) return;
    const Logits<BF16> row{static_cast<const char*>(a.logits) + r * a.stride * (BF16 ? 2 : 4), a.vocab};
    float x[Logits<BF16>::kPieces][Logits<BF16>::V];
    row.run(tile * kTile, lane, x);
    float m = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int j = 0; j < Logits<BF16>::kPieces; ++j)
#pragma unroll
        for (int e = 0; e < Logits<BF16>::V; ++e) m = fmaxf(m, x[j][e]), nan |= x[j][e] != x[j][e];
    if (nan) m = INFINITY;
    a.run_max[id * 64 + lane] = m;
    if (!s.whole(a.vocab)) return;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    double sum = 0.;
    if (m > -INFINITY && m < INFINITY) {
        const double base = m, c = s.scale();
#pragma unroll
        for (int j = 0; j < Logits<BF16>::kPieces; ++j)
#pragma unroll
            for (int e = 0; e < Logits<BF16>::V; ++e) sum += exp2_neg((static_cast<double>(x[j][e]) - base) * c);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) a.tile_sum[id] = sum;
}

// The groups of n draws, sorted in s.draw (complements of tokens).
__device__ __forceinline__ void write_groups(Shared& s, const Args& a, int r, int off, int n) {
    const int t = threadIdx.x;
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

// Draws over the tiles' prefixes in s.tile, one wave a draw: its tile, the lane in it, the token.
template <bool BF16, class F>
__device__ __forceinline__ void draw_from_tiles(Shared& s, const Args& a, const Row<BF16>& row, const Settings& set, F kept) {
    using L = Logits<BF16>;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = a.tiles;
    const double total = s.tile[tiles];
    for (int d = w; d < set.n; d += kWaves) {
        const double target = static_cast<double>(a.uniform[set.off + d]) * total;
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
        float x[L::kPieces][L::V];
        const int first = b * kTile + lane * kRun;
        row.x.consecutive(b * kTile, lane, x);
        double sum = 0.;
#pragma unroll
        for (int j = 0; j < L::kPieces; ++j)
#pragma unroll
            for (int q = 0; q < L::V; ++q) sum += kept(first + j * L::V + q, x[j][q]);
        const double incl = s.tile[b] + wave_scan(sum, lane);
        const uint64_t has = __builtin_amdgcn_ballot_w64(sum > 0.);
        const uint64_t past = has & __builtin_amdgcn_ballot_w64(incl > target);
        const int who = past ? __builtin_ctzll(past) : has ? 63 - __builtin_clzll(has) : 0;
        if (lane == who) {
            double acc = incl - sum;
            int pick = -1, last = 0;
#pragma unroll
            for (int j = 0; j < L::kPieces; ++j)
#pragma unroll
                for (int q = 0; q < L::V; ++q) {
                    const int i = first + j * L::V + q;
                    const double y = kept(i, x[j][q]);
                    acc += y;
                    if (y > 0.) {
                        last = i;
                        if (pick < 0 && acc > target) pick = i;
                    }
                }
            s.draw[d] = ~static_cast<uint32_t>(pick >= 0 ? pick : last);
        }
    }
    __syncthreads();
    write_groups(s, a, blockIdx.x, set.off, set.n);
}

// s.tile[i + 1] holds tile i's weight: makes it the prefix.
__device__ __forceinline__ void tile_prefixes(Shared& s, int tiles) {
    const int lane = threadIdx.x & 63;
    __syncthreads();
    if (threadIdx.x < 64) {
        double run = 0.;
        for (int i0 = 0; i0 < tiles; i0 += 64) {
            const double incl = run + wave_scan(i0 + lane < tiles ? s.tile[i0 + lane + 1] : 0., lane);
            if (i0 + lane < tiles) s.tile[i0 + lane + 1] = incl;
            run = __shfl(incl, 63);
        }
        if (lane == 0) s.tile[0] = 0.;
    }
    __syncthreads();
}

// Inclusive prefix sums of v (element `per` t + e of thread t) over the workgroup.
template <int per>
__device__ __forceinline__ void prefix(double (&v)[per], double* part) {
    double sum = 0., total;
#pragma unroll
    for (int e = 0; e < per; ++e) sum += v[e];
    double run = block_scan(sum, part, total);
#pragma unroll
    for (int e = 0; e < per; ++e) v[e] = run += v[e];
}

// The row's draws from the tokens above a bound on the runs' maxima; false if they are more than kList, or do not
// reach the threshold.
template <bool BF16>
__device__ bool draw_from_runs(Shared& s, const Args& a, const Row<BF16>& row, const Settings& set, const float* rm,
                               float top, float low, double whole) {
    using L = Logits<BF16>;
    const int t = threadIdx.x, n_runs = a.tiles * 64;
    const double bound = static_cast<double>(set.min_p);
    const bool by_k = set.k < a.vocab, by_p = set.p < 1.f;
    const int want = by_k ? set.k : kSparseP;
    constexpr int kHist = kBins / 2;
    // bins of equal width from the largest logit down, the last one open; wide enough for what can be drawn
    const float width = set.temp > 0.f ? fminf(top - low, 100.f * set.temp) : top - low;
    const float scale = width > 0.f ? fminf((kHist - 1) / width, 1e30f) : 0.f;
    auto bin = [&](float v) { return static_cast<int>(fminf((top - v) * scale, static_cast<float>(kHist - 1))); };
    int last = kHist - 1;
    if (by_k || by_p) {
        if (by_k && want > kSparseK) return false;
        for (int i = t; i < kHist; i += kThreads) s.hist[i] = 0;
        if (t == 0) s.i0 = kHist - 1;
        __syncthreads();
        for (int i = t; i < n_runs; i += kThreads)
            if (rm[i] > -INFINITY) atomicAdd(&s.hist[bin(rm[i])], 1u);
        __syncthreads();
        constexpr int per = kHist / kThreads;
        uint32_t c[per], sum = 0, total;
#pragma unroll
        for (int e = 0; e < per; ++e) sum += c[e] = s.hist[per * t + e];
        uint32_t run = block_scan(sum, reinterpret_cast<uint32_t*>(s.part), total);
#pragma unroll
        for (int e = 0; e < per; ++e) {
            if (run < static_cast<uint32_t>(want) && run + c[e] >= static_cast<uint32_t>(want)) s.i0 = per * t + e;
            run += c[e];
        }
        __syncthreads();
        last = s.i0;
    }
    auto above = [&](float v) { return v > -INFINITY && (by_k || by_p ? bin(v) <= last : row.weight(v) >= bound); };
    __syncthreads();
    if (t == 0) s.i1 = s.i2 = 0;
    __syncthreads();
    for (int i = t; i < n_runs; i += kThreads)
        if (above(rm[i])) {
            const int at = atomicAdd(&s.i1, 1);
            if (at < kList) s.runs[at] = i;
        }
    __syncthreads();
    const int runs = s.i1;
    if (runs > kList) return false;
    for (int i = t; i < runs * L::kPieces; i += kThreads) {
        const int run = s.runs[i / L::kPieces];
        const int first = L::token(run / 64 * kTile, run % 64, i % L::kPieces);
        float x[L::V];
        row.x.piece(first, x);
#pragma unroll
        for (int e = 0; e < L::V; ++e)
            if (above(x[e])) {
                const int at = atomicAdd(&s.i2, 1);
                if (at < kList) s.list[at] = number_of(x[e], first + e);
            }
    }
    __syncthreads();
    const int n = s.i2;
    if (n > kList) return false;
    for (int i = n + t; i < pow2_at_least(n); i += kThreads) s.list[i] = 0;
    sort_down(s.list, pow2_at_least(n));
    // weights from above, and where they are cut
    constexpr int per = kList / kThreads;
    double w[per], sum[per];
#pragma unroll
    for (int e = 0; e < per; ++e) {
        const int i = per * t + e;
        sum[e] = w[e] = i < n && i < set.k ? row.weight(logit_of(s.list[i])) : 0.;
    }
    prefix(sum, s.partd);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < per; ++e) s.cdf[per * t + e] = sum[e];
    if (t == 0) s.i0 = n < set.k ? n : set.k;
    __syncthreads();
    if (by_p) {
        const double total = by_k ? s.cdf[kList - 1] : whole, target = static_cast<double>(set.p) * total;
        if (!by_k && s.cdf[n - 1] < target) return false;
#pragma unroll
        for (int e = 0; e < per; ++e) {
            const int i = per * t + e;
            // (a run of weight 0 still holds the first token)
            if (sum[e] >= target && (i == 0 || s.cdf[i - 1] < target)) atomicMin(&s.i0, i + 1);
        }
    }
    __syncthreads();
    int keep = s.i0;
    if (bound > 0.) {
#pragma unroll
        for (int e = 0; e < per; ++e) {
            const int i = per * t + e;
            if (i > 0 && i < n && w[e] < bound) atomicMin(&s.i0, i);
        }
        __syncthreads();
        keep = s.i0;
    }
    // the kept tokens in token order, their prefixes, the draws' places among them
    const int size = pow2_at_least(keep);
    for (int i = t; i < size; i += kThreads) {
        const uint64_t x = i < keep ? s.list[i] : 0;  // (complemented index above the logit's key)
        s.list[i] = i < keep ? (x & ((1 << kIdxBits) - 1)) << 32 | x >> kIdxBits : 0;
    }
    sort_down(s.list, size);
#pragma unroll
    for (int e = 0; e < per; ++e) {
        const int i = per * t + e;
        sum[e] = i < keep ? row.weight(logit_of(s.list[i] << kIdxBits)) : 0.;
        s.hits[i] = 0;
    }
    prefix(sum, s.partd);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < per; ++e) s.cdf[per * t + e] = sum[e];
    __syncthreads();
    const double total = s.cdf[keep - 1];
    for (int d = t; d < set.n; d += kThreads) {
        const double target = static_cast<double>(a.uniform[set.off + d]) * total;
        int b = 0, e = keep;
        while (b < e) {
            const int mid = (b + e) >> 1;
            if (s.cdf[mid] > target) e = mid; else b = mid + 1;
        }
        if (b == keep) {  // none past it: the last with a weight
            b = keep - 1;
            while (b > 0 && !(s.cdf[b] > s.cdf[b - 1])) --b;
        }
        atomicAdd(&s.hits[b], 1);
    }
    __syncthreads();
    uint32_t mine = 0, groups;
#pragma unroll
    for (int e = 0; e < per; ++e) mine += s.hits[per * t + e] > 0;
    uint32_t at = block_scan(mine, reinterpret_cast<uint32_t*>(s.part), groups);
#pragma unroll
    for (int e = 0; e < per; ++e) {
        const int i = per * t + e;
        if (s.hits[i] > 0) {
            a.token[set.off + at] = (1 << kIdxBits) - 1 - static_cast<int32_t>(s.list[i] >> 32);
            a.count[set.off + at] = s.hits[i];
            ++at;
        }
    }
    if (t == 0) a.n_groups[blockIdx.x] = static_cast<int32_t>(groups);
    return true;
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void filter_draw(Args a) {
    using L = Logits<BF16>;
    __shared__ Shared s;
    const int r = blockIdx.x, t = threadIdx.x, lane = t & 63;
    const int w = __builtin_amdgcn_readfirstlane(t >> 6);
    const Settings set = settings_of(a, r);
    // (offsets are device data: a row outside the arrays reads and writes nothing)
    for (int i = t; i < set.n; i += kThreads) a.token[set.off + i] = -1, a.count[set.off + i] = 0;
    if (!set.inside || !set.valid || set.n == 0) {
        if (t == 0) a.n_groups[r] = set.inside && set.valid ? 0 : -1;
        return;
    }
    Row<BF16> row{{static_cast<const char*>(a.logits) + r * a.stride * (BF16 ? 2 : 4), a.vocab}, 0., set.scale()};
    const float* rm = a.run_max + static_cast<int64_t>(r) * a.tiles * 64;
    const double* ts = a.tile_sum + static_cast<int64_t>(r) * a.tiles;

    // the largest logit, and the smallest of the runs' largest
    float top = -INFINITY, low = INFINITY;
    for (int i = t; i < a.tiles * 64; i += kThreads) {
        const float v = rm[i];
        top = fmaxf(top, v);
        low = fminf(low, v == -INFINITY ? INFINITY : v);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o)), low = fminf(low, __shfl_xor(low, o));
    if (lane == 0) s.red[w] = top, s.red[kWaves + w] = low;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = fmaxf(top, s.red[i]), low = fminf(low, s.red[kWaves + i]);
    if (top == INFINITY || top == -INFINITY) {  // a NaN, or no distribution
        if (t == 0) a.n_groups[r] = -1;
        return;
    }
    __syncthreads();
    row.top = top;

    double whole = 0.;
    if (set.whole(a.vocab)) {
        // the tiles' weights, relative to the row's largest
        for (int i = w; i < a.tiles; i += kWaves) {
            float m = rm[i * 64 + lane];
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
            if (lane == 0) s.tile[i + 1] = m > -INFINITY ? ts[i] * row.weight(m) : 0.;
        }
        tile_prefixes(s, a.tiles);
        whole = s.tile[a.tiles];
        if (set.p >= 1.f) {
            draw_from_tiles<BF16>(s, a, row, set, [&](int, float v) { return row.weight(v); });
            return;
        }
        __syncthreads();
    }
    if (draw_from_runs<BF16>(s, a, row, set, rm, top, low, whole)) return;

    const uint64_t lo = static_cast<uint64_t>(key_of(-3.4028234663852886e38f)) << kIdxBits;
    const uint64_t hi = number_of(top, 0);
    uint64_t cut = 0;
    if (set.k < a.vocab) cut = find_cut<BF16, false>(s, row, lo, hi, static_cast<uint64_t>(set.k), 0.).number;
    if (set.p < 1.f) cut = find_cut<BF16, true>(s, row, cut > lo ? cut : lo, hi, 0, static_cast<double>(set.p)).number;
    const double bound = static_cast<double>(set.min_p);
    auto kept = [&](int i, float v) {
        const double x = row.weight(v);
        return number_of(v, i) >= cut && x >= bound ? x : 0.;
    };
    __syncthreads();
    for (int i = w; i < a.tiles; i += kWaves) {
        float x[L::kPieces][L::V];
        row.x.run(i * kTile, lane, x);
        double sum = 0.;
#pragma unroll
        for (int j = 0; j < L::kPieces; ++j)
#pragma unroll
            for (int e = 0; e < L::V; ++e) sum += kept(L::token(i * kTile, lane, j) + e, x[j][e]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        if (lane == 0) s.tile[i + 1] = sum;
    }
    tile_prefixes(s, a.tiles);
    draw_from_tiles<BF16>(s, a, row, set, kept);
}

}  // namespace

int tkv::launch_filter_sample(const FilterCall& f, void* stream) {
    Args a{};
    a.n_rows = f.n_rows, a.vocab = f.vocab, a.logits = f.logits, a.stride = f.stride;
    a.temperature = f.temperature, a.top_k = f.top_k, a.top_p = f.top_p, a.min_p = f.min_p;
    a.uniform = f.uniform, a.draw_off = f.draw_off, a.n_draws = f.n_draws;
    a.token = f.token, a.count = f.count, a.n_groups = f.n_groups;
    a.tiles = (f.vocab + kTile - 1) / kTile;
    a.tile_sum = static_cast<double*>(f.workspace);
    a.run_max = reinterpret_cast<float*>(a.tile_sum + static_cast<int64_t>(f.n_rows) * a.tiles);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    constexpr int waves = kScanThreads / 64;
    const int64_t grid = (static_cast<int64_t>(f.n_rows) * a.tiles + waves - 1) / waves;
    if (grid > INT32_MAX) return set_error(TKV_EINVAL, "tkv_filter_sample: %d rows are too many", f.n_rows);
    const auto launch = [&](auto scan, auto draw) {
        scan<<<dim3(static_cast<unsigned>(grid)), dim3(kScanThreads), 0, st>>>(a);
        draw<<<dim3(static_cast<unsigned>(f.n_rows)), dim3(kThreads), 0, st>>>(a);
    };
    if (f.logit_type == TKV_LOGITS_BF16)
        launch(filter_scan<true>, filter_draw<true>);
    else
        launch(filter_scan<false>, filter_draw<false>);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TKV_OK : set_error(TKV_EHIP, "tkv_filter_sample launch: %s", hipGetErrorString(e));
}
