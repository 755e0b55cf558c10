// Draws from a truncated temperature softmax, with settings for each row (tkv_filter_sample).
//
// Tokens are ordered by (logit descending, index ascending), here as one 53-bit number a token: the logit's bits,
// mapped so that larger means larger, above the complement of the index.  All numbers of a row differ, and what
// top-k, top-p and min-p keep is everything from a threshold up, so truncation is finding that threshold:
//   top-k   the k-th number from above;
//   top-p   the number at which the sum of the weights from above reaches top_p times the (top-k) total;
//   min-p   a bound on the weight itself.
//
// filter_scan streams the logits once, a wave per tile of 2,048: the largest logit of every run of 32 and, for rows whose
// whole weight is asked for (top-p without top-k, or no truncation), the weights of the tile's parts (64 lanes x 16
// bytes: 512 tokens of bf16, 256 of fp32) relative to the tile's largest logit, and a sample of two logits a run.
// filter_draw takes a workgroup a row.  The runs' maxima bound the threshold from below (the k-th largest of them is at
// most the k-th largest logit), so only the few runs above that bound are read again, their tokens above it sorted, cut
// and drawn from.  For top-p the bound comes from the sample, which tells how much weight lies below a logit to a few
// per cent.
// Where thousands of tokens are kept the row goes through two more kernels, which find nothing to do otherwise:
// filter_narrow reads it again, a wave a tile, for the weight above the interval that must hold the threshold and the
// numbers inside it (top-k: all from the interval's end up, which by the sample are k and a few), and filter_finish cuts
// among those and draws.  A row that slips through (more tokens at the threshold than a list holds, a top-k of more than
// half a list, a threshold outside the interval) is read by one workgroup as often as it takes: histograms over the
// numbers, 2,048 bins of the interval that still holds the threshold, with each bin's count and weight, until that
// interval holds few enough tokens to sort.  The sample's positions are fixed, so a row whose logits follow them goes this
// way: 8 rows of 151,936 under a top-p of 0.9 take 48 us, 259 where the sampled tokens lie 30 below the others and 227 where
// they lie 4 above; 100 rows 84, 313 and 288.
//
// Weights are computed in fp64, w = 2^((l - max) log2(e) / T), and summed in a fixed order.  Histogram sums are
// integers, w in units of 2^-42, so that they do not depend on the order of the atomics; they decide where top-p ends
// to 2^-43 of the largest weight a token.
//
// What bounds it (MI355X).  The scan: memory, 608 MB of fp32 logits (1,000 rows of 151,936) in 98 to 107 us, 5.7 to 6.2 TB/s,
// past the caches; where a third of the rows ask for their whole weight the fp64 exponentials (ten FMAs each) hide behind it.
// The draw: latency, one workgroup's chain of barriers, 14 us for 5 rows, 25 us for 250 (a workgroup a CU), 42 us for
// 1,000 (three on a CU at once).  filter_narrow and filter_finish find nothing in 2 to 4 and 1.6 us; 136 rows of the 1,000
// take them 42 and 31 us: a second read of 83 MB with an exponential for each logit above the interval, then 20 us of one
// workgroup's chain (a list of some thousand numbers weighed, a histogram, a sort, the draws).
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cstdint>

#include "internal.h"

namespace {

constexpr int kThreads = 512;         // a row's workgroup
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kList = 2048;           // tokens that are sorted
constexpr int kIdxBits = 21;          // vocabularies of up to 2^21 tokens
constexpr int kRun = 32;              // consecutive tokens whose largest logit is kept
constexpr int kTile = tkv::kFilterTile;
static_assert(kTile == 64 * kRun, "as many runs as lanes");
constexpr int kScanThreads = 256;
constexpr int kSparseP = 64;          // fewest runs looked into for top-p
constexpr int kSparseRuns = 1024;     // most runs that are looked into for top-k
constexpr int kSparseFew = 384;       // and for top-p and min-p, past which filter_narrow reads the row; within 3% whatever it is
                                      // (250 rows of 152,064 101 us, 192: 100, 768: 101; 333 of 32,003 90, 88 and 90; 1,000 of
                                      // 151,936 230, 236, 230)
constexpr int kSparseK = 512;         // largest top-k that they are looked into for where a list holds twice as many numbers:
                                      // 8 rows of 151,936 under a top-k of 500 31 us, 44 by the sample; of 1,000 41 and 45.
                                      // 200 rows of 32,000 (1,000 runs) under a top-k of 1,000 112 and 49, of 151,936 59 and
                                      // 87, but where a few do and others keep thousands of tokens anyway 101 and 85
constexpr int kHist = 1024;           // bins of the runs' maxima and of the sample
constexpr int kMaxTiles = (1 << kIdxBits) / kTile;
constexpr int kMaxPotential = 1024;
constexpr double kUnit = 4398046511104.0;     // 2^42: units of weights that histograms add up (2^21 of 1 at most)
constexpr double kFine = 1125899906842624.0;  // 2^50: of a list's kept weights (8,192 of 1 at most)

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
    int32_t tiles, cap;   // a row's tiles; numbers its list holds
    int32_t* n_again;     // rows that are read again, and which
    struct Again* again;
    float2* tile_max;                 // [n_rows][tiles]: the largest logit, the smallest that filter_draw's bins are to hold
    float *run_max, *sample;          // [n_rows][tiles][64], sample: two of them
    double* part_sum;                 // [n_rows][tiles][8]: weight of a tile's parts relative to the tile's largest logit
    double *above, *kept;             // [n_rows][tiles] and its parts: filter_narrow's
    uint64_t* lists;                  // [n_rows][cap]
};

// A row that is read again.  The interval that holds its threshold is bins [first, last] of equal width below the
// largest logit.
struct Again {
    int32_t row, whole_row;  // whole_row: by one workgroup
    int32_t first, last;
    float top, scale;
    double weight;           // of all tokens, if top-p is to be cut
    int32_t n;               // numbers inside the interval
    int32_t pad[3];
};
static_assert(sizeof(Again) == 48, "the workspace's records");

// Bins of equal width from the largest logit down, the last one open.
__device__ __forceinline__ int bin_of(float v, float top, float scale) {
    return static_cast<int>(fminf(fminf(top - v, 3.4028234663852886e38f) * scale, static_cast<float>(kHist - 1)));
}

// A row's settings and draws.
struct Settings {
    float temp, p, min_p;
    int k;        // vocab: all
    int off, n;
    bool inside;  // its draws are inside the arrays
    bool valid;
    // the weight of all of the row's tokens decides something
    __device__ __forceinline__ bool whole(int vocab) const { return k >= vocab && (p < 1.f || min_p <= 0.f); }
    // top-k by a sample: too many runs would hold some of the k tokens
    __device__ __forceinline__ bool many(int vocab, int cap) const { return k < vocab && k > kSparseK && 2 * static_cast<int64_t>(k) <= cap; }
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
    // (by their bits: the compiler may assume that a number is no NaN)
    const auto below = [](float v, uint32_t end) { return __float_as_uint(v) == 0x80000000u || __float_as_uint(v) < end; };
    s.valid = below(s.temp, 0x7f800000u) && below(s.p, 0x3f800001u) && below(s.min_p, 0x3f800001u) && s.k >= 0;
    if (s.temp == 0.f) s.k = 1;
    if (s.k == 0 || s.k > a.vocab) s.k = a.vocab;
    return s;
}

// 2^t for t <= 0, to 2^-50: t's nearest integer n by adding 1.5 * 2^52, and 2^(t - n) as 1 + f p(f), p the polynomial
// that meets (2^f - 1) / f at ten Chebyshev nodes of [-1/2, 1/2].  (2^0 is 1 exactly: equal logits have equal sums.)
__device__ __forceinline__ double exp2_neg(double t) {
    constexpr double kRound = 6755399441055744.0;
    t = fmax(t, -1100.);
    const double r = t + kRound;
    const int n = static_cast<int>(__double_as_longlong(r));
    const double f = t - (r - kRound);
    double y = 0x1.e5e9f548e5725p-28;
    y = fma(y, f, 0x1.b6571de2f2351p-24);
    y = fma(y, f, 0x1.62bfe46117445p-20);
    y = fma(y, f, 0x1.ffcb76789860fp-17);
    y = fma(y, f, 0x1.4309130378460p-13);
    y = fma(y, f, 0x1.5d87fe908f88ap-10);
    y = fma(y, f, 0x1.3b2ab6fba385fp-7);
    y = fma(y, f, 0x1.c6b08d7044119p-5);
    y = fma(y, f, 0x1.ebfbdff82c590p-3);
    y = fma(y, f, 0x1.62e42fefa39f7p-1);
    y = fma(y, f, 1.);
    return __builtin_amdgcn_ldexp(y, n);
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
    // this lane's tokens of the tile that starts at a0: kPieces pieces of V tokens, 64 V apart (-inf past the row)
    // (a piece of all 64 lanes is a part of the tile, consecutive tokens; kPieces lanes of one are a run)
    static constexpr int V = BF16 ? 8 : 4, kPieces = kRun / V;
    static __device__ __forceinline__ int token(int a0, int lane, int piece) { return a0 + (piece * 64 + lane) * V; }
    // the first of the `sub`-th V tokens of run r
    static __device__ __forceinline__ int token_of_run(int r, int sub) {
        const int in = r % 64;
        return token(r / 64 * kTile, in / kPieces * kPieces + sub, in % kPieces);
    }
    template <bool NT = false>
    __device__ __forceinline__ void piece(int a, float (&x)[V]) const {
        if (a + V <= vocab) {
            if constexpr (BF16) {
                const u16x8_t* from = reinterpret_cast<const u16x8_t*>(static_cast<const uint16_t*>(p) + a);
                const u16x8_t y = NT ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = bf16_f32(y[e]);
            } else {
                const f32x4_t* from = reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p) + a);
                const f32x4_t y = NT ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = y[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = a + e < vocab ? at(a + e) : -INFINITY;
        }
    }
    template <bool NT = false>
    __device__ __forceinline__ void tile(int a0, int lane, float (&x)[kPieces][V]) const {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) piece<NT>(token(a0, lane, j), x[j]);
    }
};

// Sums of v[0], v[1], .. over the wave, in a fixed pattern: lane 64 / N j .. 64 / N (j + 1) - 1 gets v[j]'s.
template <int N, int O = 32>
__device__ __forceinline__ double wave_sums(const double (&v)[N], int lane) {
    if constexpr (N > 1) {
        const bool upper = lane & O;
        double u[N / 2];
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            const double mine = upper ? v[j + N / 2] : v[j], other = upper ? v[j] : v[j + N / 2];
            u[j] = mine + __shfl_xor(other, O);
        }
        return wave_sums<N / 2, O / 2>(u, lane);
    } else {
        double sum = v[0];
#pragma unroll
        for (int o = O; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        return sum;
    }
}

// v of another lane by a data-parallel move (within a row of 16, or a row's last lane to the rows behind), `none` where
// that lane does not exist or the row is not in ROWS.
template <int CTRL, int ROWS, class T>
__device__ __forceinline__ T moved(T v, T none) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
    } else {
        const int2 x = __builtin_bit_cast(int2, v), n = __builtin_bit_cast(int2, none);
        return __builtin_bit_cast(T, int2{__builtin_amdgcn_update_dpp(n.x, x.x, CTRL, ROWS, 0xf, false),
                                          __builtin_amdgcn_update_dpp(n.y, x.y, CTRL, ROWS, 0xf, false)});
    }
}
// Inclusive scan over a wave (all lanes there), in a fixed pattern: within rows of 16, then the rows before.
template <class T, class Op>
__device__ __forceinline__ T wave_scan(T v, T none, Op op) {
    v = op(v, moved<0x111, 0xf>(v, none));
    v = op(v, moved<0x112, 0xf>(v, none));
    v = op(v, moved<0x114, 0xf>(v, none));
    v = op(v, moved<0x118, 0xf>(v, none));
    v = op(v, moved<0x142, 0xa>(v, none));  // lane 15 to row 1, lane 47 to row 3
    return op(v, moved<0x143, 0xc>(v, none));  // lane 31 to rows 2 and 3
}
template <class T>
__device__ __forceinline__ T wave_scan(T v) {
    return wave_scan(v, T{0}, [](T a, T b) { return a + b; });
}
// v of one lane, for all.
template <class T>
__device__ __forceinline__ T lane_of(T v, int lane) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    } else {
        const int2 x = __builtin_bit_cast(int2, v);
        return __builtin_bit_cast(T, int2{__builtin_amdgcn_readlane(x.x, lane), __builtin_amdgcn_readlane(x.y, lane)});
    }
}
__device__ __forceinline__ float wave_max(float v) {
    return lane_of(wave_scan(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); }), 63);
}
__device__ __forceinline__ int wave_max(int v) {
    return lane_of(wave_scan(v, INT32_MIN, [](int a, int b) { return a > b ? a : b; }), 63);
}

// Exclusive scan over the workgroup and the total; `part` holds a value a wave.
template <class T>
__device__ __forceinline__ T block_scan(T v, T* part, T& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const T incl = wave_scan(v);
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

// v of the lane whose index differs in one bit.
__device__ __forceinline__ uint32_t lane_xor(uint32_t v, int bit) { return static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), bit)); }
__device__ __forceinline__ uint64_t lane_xor(uint64_t v, int bit) {
    return static_cast<uint64_t>(lane_xor(static_cast<uint32_t>(v >> 32), bit)) << 32 | lane_xor(static_cast<uint32_t>(v), bit);
}

// Bitonic sort of E * kThreads numbers, descending, in registers: number e * kThreads + t is thread t's.  Pairs within a
// wave go over the lanes, pairs within a thread stay, the rest go through LDS.
template <int E, class T>
__device__ __forceinline__ void sort_registers(T* a) {
    const int t = threadIdx.x;
    T x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = a[e * kThreads + t];
#pragma unroll 1
    for (int k = 2; k <= E * kThreads; k <<= 1) {
        int j = k >> 1;
#pragma unroll
        for (int d = E / 2; d > 0; d >>= 1)
            if (j == d * kThreads) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if ((e & d) == 0) {
                        const bool down = ((e * kThreads + t) & k) == 0;
                        const T p = x[e], q = x[e + d];
                        if ((p < q) == down) x[e] = q, x[e + d] = p;
                    }
                j >>= 1;
            }
#pragma unroll 1
        for (; j >= 64; j >>= 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) a[e * kThreads + t] = x[e];
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const T y = a[e * kThreads + (t ^ j)];
                const bool larger = ((t & j) == 0) == (((e * kThreads + t) & k) == 0);
                x[e] = (x[e] < y) == larger ? y : x[e];
            }
        }
#pragma unroll 1
        for (; j > 0; j >>= 1) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const T y = lane_xor(x[e], j);
                const bool larger = ((t & j) == 0) == (((e * kThreads + t) & k) == 0);
                x[e] = (x[e] < y) == larger ? y : x[e];
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) a[e * kThreads + t] = x[e];
    __syncthreads();
}

// Sorts n numbers (0 is none), descending; a has room for the next multiple of kThreads.  Few are counted: each
// thread those before its own.
template <class T>
__device__ __forceinline__ void sort_down(T* a, int n) {
    constexpr int kCounted = 256;
    const int t = threadIdx.x;
    static_assert(kList == 8 * kThreads || kList == 4 * kThreads, "the sizes below");
    int size = (n + 63) & ~63;
    if (n > kCounted)
        for (size = kThreads; size < n;) size *= 2;
    for (int i = n + t; i < size; i += kThreads) a[i] = 0;
    __syncthreads();
    if (n <= kCounted) {
        // `parts` threads a number, each over its share of the others, 16 in flight
        const int parts = kThreads / (n <= 128 ? 128 : 256), i = t / parts, share = size / parts, from = (t & (parts - 1)) * share;
        const T mine = i < n ? a[i] : 0;
        int rank = 0;
        constexpr int P = 16 / sizeof(T);
        typedef T pack_t __attribute__((ext_vector_type(P)));
        for (int q = from; q < from + share; q += 16) {
            pack_t v[16 / P];
#pragma unroll
            for (int e = 0; e < 16 / P; ++e) v[e] = *reinterpret_cast<const pack_t*>(a + q + e * P);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const T other = v[e / P][e % P];
                rank += other > mine;
                if constexpr (sizeof(T) == 4) rank += other == mine && q + e < i;  // (only draws repeat)
            }
        }
        for (int o = parts / 2; o > 0; o >>= 1) rank += __shfl_xor(rank, o);
        __syncthreads();
        if (i < n && (t & (parts - 1)) == 0) a[rank] = mine;
        __syncthreads();
    } else if (size == kThreads) {
        sort_registers<1>(a);
    } else if (size == 2 * kThreads) {
        sort_registers<2>(a);
    } else if (size == 4 * kThreads) {
        sort_registers<4>(a);
    } else {
        sort_registers<kList / kThreads>(a);
    }
}

struct __attribute__((aligned(16))) Shared {
    union {
        struct {
            uint64_t mass[kBins];
            uint32_t cnt[kBins];
        } h;
        struct {
            uint64_t list[kList];  // the tokens above the bound
            union {
                struct {
                    uint32_t hist[kHist], sampled[kHist];
                    int32_t runs[kSparseRuns];
                };
                double cdf[kList];
            };
            uint32_t hits[kList / 2];  // draws of each kept token, 16 bits each
        };
        struct {
            double tile[kMaxTiles + 1];   // the draws' tile prefixes
            double want[kMaxPotential];   // each draw's target past its part's start
            uint32_t found[kMaxPotential];  // and its token's complement
        };
    };
    uint64_t part[kWaves];
    double partd[kWaves];
    union {
        __attribute__((aligned(16))) uint32_t draw[kMaxPotential];  // complements of the tokens drawn
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

// Sources of numbers: a whole row, or a list.
template <bool BF16>
struct RowNumbers {
    Logits<BF16> x;
    template <class F>
    __device__ __forceinline__ void each(F f) const {
        x.each([&](int i, float v) { f(number_of(v, i), uint64_t{0}); });
    }
};
// (in registers, with each number's weight in units; 0 is none)
constexpr int kMine = 8192 / kThreads;
struct ListNumbers {
    uint64_t n[kMine], w[kMine];
    template <class F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int e = 0; e < kMine; ++e)
            if (n[e] != 0) f(n[e], w[e]);
    }
};

// The last number of the shortest run from above that reaches a target, among a source's numbers in [lo, hi]; lo if all
// of them do not.  by_mass: the target is `want` units of weight, or (share) that share of the whole weight in [lo, hi];
// else a count.
// fresh(logit): a token's weight, where the source has none.
template <class Src, class W>
__device__ __forceinline__ uint64_t find_cut(Shared& s, const Src& src, const W& fresh, bool by_mass, bool share, uint64_t lo, uint64_t hi, uint64_t target,
                                             double want) {
    const int t = threadIdx.x;
    uint64_t above_c = 0, above_m = 0;
    const uint64_t floor = lo;
    const auto units = [&](uint64_t n, uint64_t w) { return w != 0 ? w : fresh(logit_of(n)); };
    for (bool first = true;; first = false) {
        const int bits = 64 - __builtin_clzll(hi - lo | 1), shift = bits > 11 ? bits - 11 : 0;
        __syncthreads();
        for (int i = t; i < kBins; i += kThreads) s.h.mass[i] = 0, s.h.cnt[i] = 0;
        __syncthreads();
        src.each([&](uint64_t n, uint64_t w) {
            if (n < lo || n > hi) return;
            const int b = static_cast<int>((n - lo) >> shift);
            atomicAdd(&s.h.cnt[b], 1u);
            if (by_mass) atomicAdd(reinterpret_cast<unsigned long long*>(&s.h.mass[b]), static_cast<unsigned long long>(units(n, w)));
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
        if (share && first) want *= static_cast<double>(total_m);
        if (t == 0) s.i0 = -1;
        __syncthreads();
        uint64_t bc = before_c, bm = before_m;
#pragma unroll
        for (int e = 0; e < per; ++e) {
            const uint64_t ac = bc + c[e], am = bm + m[e];
            const bool reached = by_mass ? static_cast<double>(am) >= want : ac >= target;
            const bool was = by_mass ? static_cast<double>(bm) >= want : bc >= target;
            // (the first bin that holds anything, if nothing is wanted)
            if (c[e] > 0 && reached && (!was || bc == 0)) {
                s.i0 = kBins - 1 - (per * t + e);
                s.i1 = static_cast<int>(c[e]);
                s.u0 = bc, s.u1 = bm;
            }
            bc = ac, bm = am;
        }
        __syncthreads();
        if (s.i0 < 0) return floor;  // all of it is less than the target
        const int bin = s.i0, n = s.i1;
        above_c = s.u0, above_m = s.u1;
        lo += static_cast<uint64_t>(bin) << shift;
        hi = lo + ((uint64_t{1} << shift) - 1);
        if (n > kList) continue;
        // few enough to sort
        __syncthreads();
        if (t == 0) s.i0 = 0;
        __syncthreads();
        src.each([&](uint64_t x, uint64_t) {
            if (x >= lo && x <= hi) s.list[atomicAdd(&s.i0, 1)] = x;
        });
        sort_down(s.list, n);
        constexpr int many = kList / kThreads;
        uint64_t mine = 0, total, w[many];
#pragma unroll
        for (int e = 0; e < many; ++e) {
            const int i = many * t + e;
            mine += w[e] = by_mass && i < n ? fresh(logit_of(s.list[i])) : 0;
        }
        uint64_t run = above_m + block_scan(mine, s.part, total);
        if (t == 0) s.u0 = s.list[n - 1];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < many; ++e) {
            const int i = many * t + e;
            const uint64_t next = run + w[e];
            const bool reached = by_mass ? static_cast<double>(next) >= want : above_c + i + 1 >= target;
            const bool was = by_mass ? static_cast<double>(run) >= want : above_c + i >= target;
            if (i < n && reached && (!was || above_c + i == 0)) s.u0 = s.list[i];
            run = next;
        }
        __syncthreads();
        const uint64_t cut = s.u0;
        __syncthreads();
        return cut;
    }
}

// A wave a tile: the runs' maxima (+inf where a logit is NaN), and the parts' weights where the row asks for them.
// NT: logits are read past the caches, from 192 MiB on.  The whole call on logits just written, read through and past:
// 61 MB 75 and 76 us, 152 MB 104 and 105, 243 MB 142 and 135, 365 MB 226 and 198, 608 MB 338 and 306.
template <bool BF16, bool NT>
__global__ __launch_bounds__(kScanThreads) __attribute__((amdgpu_waves_per_eu(5))) void filter_scan(Args a) {
    const int lane = threadIdx.x & 63;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * (kScanThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = static_cast<int>(id / a.tiles), tile = static_cast<int>(id - static_cast<int64_t>(r) * a.tiles);
    if (id == 0 && lane == 0) *a.n_again = 0;
    if (r >= a.n_rows) return;
    const Settings s = settings_of(a, r);
    if (!s.inside || !s.valid || s.n == 0) return;
    const Logits<BF16> row{static_cast<const char*>(a.logits) + r * a.stride * (BF16 ? 2 : 4), a.vocab};
    float x[Logits<BF16>::kPieces][Logits<BF16>::V];
    row.template tile<NT>(tile * kTile, lane, x);
    // Run l is piece l % N of the lanes l / N * N .. + N - 1 (consecutive tokens, so that filter_draw reads few lines; a
    // lane's own pieces as a run cost this kernel 4 us less of 102 and filter_draw 6 to 12 more).  The N pieces' maxima over
    // N lanes by halving: each exchange leaves a lane half of the pieces over twice the lanes.
    constexpr int N = Logits<BF16>::kPieces;
    float p[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        p[j] = -INFINITY;
        bool nan = false;
#pragma unroll
        for (int e = 0; e < Logits<BF16>::V; ++e) p[j] = fmaxf(p[j], x[j][e]), nan |= (__float_as_uint(x[j][e]) & 0x7fffffffu) > 0x7f800000u;
        if (nan) p[j] = INFINITY;
    }
    if constexpr (N == 8) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float keep = lane & 4 ? p[j + 4] : p[j], give = lane & 4 ? p[j] : p[j + 4];
            p[j] = fmaxf(keep, moved<0x141, 0xf>(give, -INFINITY));  // lane 7 - l of eight
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float keep = lane & 2 ? p[j + 2] : p[j], give = lane & 2 ? p[j] : p[j + 2];
        p[j] = fmaxf(keep, moved<0x4e, 0xf>(give, -INFINITY));  // quad_perm 2 3 0 1
    }
    float m = fmaxf(lane & 1 ? p[1] : p[0], moved<0xb1, 0xf>(lane & 1 ? p[0] : p[1], -INFINITY));  // quad_perm 1 0 3 2
    a.run_max[id * 64 + lane] = m;
    const bool whole = s.whole(a.vocab), samples = (whole && s.p < 1.f) || s.many(a.vocab, a.cap);
    const float s0 = x[0][0], s1 = x[Logits<BF16>::kPieces / 2][0];
    if (samples) a.sample[id * 128 + lane] = s0, a.sample[id * 128 + 64 + lane] = s1;
    const auto finite = [](float v) { return v == -INFINITY ? INFINITY : v; };
    float low = samples ? fminf(finite(s0), finite(s1)) : finite(m);
    m = wave_max(m), low = -wave_max(-low);
    if (lane == 0) a.tile_max[id] = make_float2(m, low);
    if (!whole) return;
    double sum[N];
    const bool some = m > -INFINITY && m < INFINITY;
    const double base = some ? m : 0., c = s.scale();
#pragma unroll
    for (int j = 0; j < N; ++j) {
        sum[j] = 0.;
        if (some)
#pragma unroll
            for (int e = 0; e < Logits<BF16>::V; ++e) sum[j] += exp2_neg((static_cast<double>(x[j][e]) - base) * c);
    }
    const double part = wave_sums(sum, lane);
    if (lane % (64 / N) == 0) a.part_sum[id * N + lane / (64 / N)] = part;
}

// The groups of n draws, sorted in s.draw (complements of tokens).
__device__ __forceinline__ void write_groups(Shared& s, const Args& a, int r, int off, int n) {
    const int t = threadIdx.x;
    sort_down(s.draw, n);
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

// Draws over the tiles' prefixes in s.tile, and the parts' weights part(tile, j).  A sum that rounding leaves short of the
// target falls to the last one with a weight.
template <bool BF16, class P, class F>
__device__ __forceinline__ void draw_from_tiles(Shared& s, const Args& a, int r, const Row<BF16>& row, const Settings& set, P part, F kept) {
    using L = Logits<BF16>;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = a.tiles;
    const double total = s.tile[tiles];
    // a thread a draw: its tile and part
    for (int d = threadIdx.x; d < set.n; d += kThreads) {
        // (at least 2^-1000, total being 1 or more: a uniform of 0 passes over a tile whose weight is positive only as a
        // sum, its tokens' own weights having rounded to 0)
        const double target = fmax(static_cast<double>(a.uniform[set.off + d]) * total, 0x1p-1000);
        int b = 0, e = tiles;  // the first tile that ends past the target
        while (b < e) {
            const int mid = (b + e) >> 1;
            if (s.tile[mid + 1] > target) e = mid; else b = mid + 1;
        }
        if (b == tiles) {  // none: the last with a weight
            b = tiles - 1;
            while (b > 0 && !(s.tile[b + 1] > s.tile[b])) --b;
        }
        double weight[L::kPieces], run = s.tile[b], start = run;
#pragma unroll
        for (int j = 0; j < L::kPieces; ++j) weight[j] = part(b, j);
        int in = 0;
        bool past = false;
#pragma unroll
        for (int j = 0; j < L::kPieces; ++j) {
            if (!past && weight[j] > 0.) in = j, start = run;
            run += weight[j];
            past = past || (weight[j] > 0. && run > target);
        }
        s.draw[d] = static_cast<uint32_t>(b * L::kPieces + in);
        s.want[d] = target - start;
    }
    __syncthreads();
    // a wave a draw, two on their way at once: the lane that has it, and the token
    constexpr int kAtOnce = 2;
    for (int d0 = w; d0 < set.n; d0 += kAtOnce * kWaves) {
        int first[kAtOnce];
        float x[kAtOnce][L::V];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int p = __builtin_amdgcn_readfirstlane(static_cast<int>(s.draw[min(d0 + u * kWaves, set.n - 1)]));
            first[u] = (p * 64 + lane) * L::V;
            row.x.piece(first[u], x[u]);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int d = d0 + u * kWaves;
            if (d >= set.n) break;
            const double target = s.want[d];
            double y[L::V], sum = 0.;
#pragma unroll
            for (int q = 0; q < L::V; ++q) sum += y[q] = kept(first[u] + q, x[u][q]);
            const double incl = wave_scan(sum);
            const uint64_t has = __builtin_amdgcn_ballot_w64(sum > 0.);
            const uint64_t past = has & __builtin_amdgcn_ballot_w64(incl > target);
            const int who = past ? __builtin_ctzll(past) : has ? 63 - __builtin_clzll(has) : 0;
            if (lane == who) {
                double acc = incl - sum;
                int pick = -1, last = 0;
#pragma unroll
                for (int q = 0; q < L::V; ++q) {
                    acc += y[q];
                    if (y[q] > 0.) {
                        last = first[u] + q;
                        if (pick < 0 && acc > target) pick = last;
                    }
                }
                s.found[d] = ~static_cast<uint32_t>(pick >= 0 ? pick : last);
            }
        }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < set.n; d += kThreads) s.draw[d] = s.found[d];
    __syncthreads();
    write_groups(s, a, r, set.off, set.n);
}

// s.tile[i + 1] holds tile i's weight: makes it the prefix.
__device__ __forceinline__ void tile_prefixes(Shared& s, int tiles) {
    const int lane = threadIdx.x & 63;
    __syncthreads();
    if (threadIdx.x < 64) {
        double run = 0.;
        for (int i0 = 0; i0 < tiles; i0 += 64) {
            const double incl = run + wave_scan(i0 + lane < tiles ? s.tile[i0 + lane + 1] : 0.);
            if (i0 + lane < tiles) s.tile[i0 + lane + 1] = incl;
            run = lane_of(incl, 63);
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

// Room for this lane's set bits behind what `counter` counts, with one atomic for the wave's lanes that are here.
__device__ __forceinline__ int append(int* counter, uint32_t bits) {
    const int mine = __builtin_popcount(bits);
    int before = 0, total = 0;
    const uint64_t here = __builtin_amdgcn_ballot_w64(true);
    // (bit by bit of the counts, which are at most 32)
#pragma unroll
    for (int k = 0; k < 6; ++k) {
        const uint64_t b = __builtin_amdgcn_ballot_w64(mine >> k & 1);
        before += static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(b >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(b), 0))) << k;
        total += __builtin_popcountll(b) << k;
    }
    int base = 0;
    const int leader = __builtin_ctzll(here);
    if (static_cast<int>(threadIdx.x & 63) == leader && total > 0) base = atomicAdd(counter, total);
    return __builtin_amdgcn_readlane(base, leader) + before;
}

// f(i, p[i]) for i < n, eight loads ahead.
template <class F>
__device__ __forceinline__ void each_of(const float* p, int n, F f) {
    for (int i0 = threadIdx.x; i0 < n; i0 += 8 * kThreads) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = p[min(i0 + e * kThreads, n - 1)];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i0 + e * kThreads < n) f(i0 + e * kThreads, v[e]);
    }
}

// What is to be looked at of a row: the tokens from a logit up.
struct Bound {
    float low;
    bool min_p;       // all that min-p keeps are among them, wherever top-p ends
    int first, last;  // the bins that may hold the threshold
    int runs;         // runs that hold some of the tokens
};
// A logit in or below a bin, by a little (all for the last bin).
__device__ __forceinline__ float foot_of(int bin, float top, float scale) {
    return bin >= kHist - 1 || scale == 0.f ? -3.4028234663852886e38f : top - (bin + 1.01f) / scale;
}

// The bound for a row that top-k or top-p cuts.
template <bool BF16>
__device__ Bound find_bound(Shared& s, const Args& a, const Row<BF16>& row, const Settings& set, const float* rm, const float* sample,
                            float top, float scale, double whole) {
    const int t = threadIdx.x, n_runs = a.tiles * 64;
    const bool by_k = set.k < a.vocab, sampled = !by_k || set.many(a.vocab, a.cap);
    const uint32_t want = by_k ? set.k : kSparseP;
    constexpr int per = kHist / kThreads;
    for (int i = t; i < kHist; i += kThreads) s.hist[i] = 0, s.sampled[i] = 0;
    if (t == 0) s.i0 = kHist - 1, s.i1 = s.i2 = by_k ? kHist - 1 : -1;
    __syncthreads();
    each_of(rm, n_runs, [&](int, float v) {
        if (v > -INFINITY) atomicAdd(&s.hist[bin_of(v, top, scale)], 1u);
    });
    // (positions past the row hold -inf)
    if (sampled)
        each_of(sample, 2 * n_runs, [&](int, float v) {
            if (v > -INFINITY) atomicAdd(&s.sampled[bin_of(v, top, scale)], 1u);
        });
    __syncthreads();
    uint32_t c[per], sum = 0, total;
#pragma unroll
    for (int e = 0; e < per; ++e) sum += c[e] = s.hist[per * t + e];
    uint32_t run = block_scan(sum, reinterpret_cast<uint32_t*>(s.part), total);
#pragma unroll
    for (int e = 0; e < per; ++e) {
        if (run < want && run + c[e] >= want) s.i0 = per * t + e;
        run += c[e];
        s.hist[per * t + e] = run;  // runs up to this bin
    }
    constexpr int V = Logits<BF16>::V;
    const int left = a.vocab - (a.tiles - 1) * kTile;
    const int n_sampled = (a.tiles - 1) * 128 + min(64, (left + V - 1) / V) + max(0, min(64, (left - kTile / 2 + V - 1) / V));
    const double each = static_cast<double>(a.vocab) / n_sampled;  // tokens that a sampled one stands for
    if (by_k && sampled) {
        // the bin from which on, by the sample and four standard errors of it, there are k tokens
        uint32_t c[per], sum = 0, total;
#pragma unroll
        for (int e = 0; e < per; ++e) sum += c[e] = s.sampled[per * t + e];
        uint32_t run = block_scan(sum, reinterpret_cast<uint32_t*>(s.part), total);
        const float most = static_cast<float>(set.k / each);
        const auto enough = [&](uint32_t n) { return static_cast<float>(n) - 4.f * sqrtf(static_cast<float>(n)) >= most; };
#pragma unroll
        for (int e = 0; e < per; ++e) {
            if (!enough(run) && enough(run + c[e])) s.i1 = per * t + e;
            run += c[e];
        }
    }
    if (!by_k) {
        // From the smallest logit up (thread t takes bins kHist - 1 - per t and the next above): the weight below a
        // bin's upper edge, estimated from the sample, and its standard error; both by the weight at the bin's middle.
        // The largest of them may be wide off (few tokens, much weight): what matters is where it passes `rest`.
        const double rest = (1. - static_cast<double>(set.p)) * whole;
        const double slope = scale > 0.f ? -row.c / static_cast<double>(scale) : 0.;
        double m[per], v[per], ms = 0., vs = 0., all;
        uint32_t cs = 0, every;
#pragma unroll
        for (int e = 0; e < per; ++e) {
            const int b = kHist - 1 - (per * t + e);
            const double w = each * exp2_neg((b + .5) * slope);
            ms += m[e] = w * s.sampled[b];
            vs += v[e] = w * w * s.sampled[b];
            cs += c[e] = s.sampled[b];
        }
        uint32_t crun = block_scan(cs, reinterpret_cast<uint32_t*>(s.part), every);
        double mrun = block_scan(ms, s.partd, all);
        double vrun = block_scan(vs, s.partd, all);
        int may = -1, must = -1;
#pragma unroll
        for (int e = 0; e < per; ++e) {
            const int b = kHist - 1 - (per * t + e);
            mrun += m[e], vrun += v[e];
            const double err = 4. * sqrt(vrun) + 4. * each * exp2_neg(b * slope);
            if (mrun + err >= rest) may = max(may, b);   // the last bin that may hold the threshold: past it there is too little
            if (mrun - err > rest) must = max(must, b);  // the first: from it on there is too much
            s.sampled[b] = every - crun;                 // samples in bins above
            crun += c[e];
        }
        may = wave_max(may), must = wave_max(must);
        if ((t & 63) == 0) atomicMax(&s.i1, may), atomicMax(&s.i2, must);
    }
    __syncthreads();
    Bound r{};
    r.last = s.i0, r.first = 0;
    if (by_k && sampled) r.last = min(r.last, s.i1);
    if (!by_k) {
        r.last = max(s.i0, min(s.i1 + 1, kHist - 1));
        r.first = max(0, s.i2 - 1);
    }
    r.runs = s.hist[r.last];
    r.low = foot_of(r.last, top, scale);
    // (a sampled token stands for 16)
    if (sampled && (by_k || r.runs > kSparseFew || 16 * s.sampled[r.last] > kSparseFew)) r.runs = kSparseRuns + 1;
    __syncthreads();
    return r;
}

// The row's draws from the tokens above a bound; false if they are more than kList, or do not reach the threshold (waves may
// then still be reading `s`).
template <bool BF16>
__device__ bool draw_from_runs(Shared& s, const Args& a, int r, const Row<BF16>& row, const Settings& set, const float* rm,
                               double whole, const Bound& at_least) {
    using L = Logits<BF16>;
    const int t = threadIdx.x, n_runs = a.tiles * 64;
    const double bound = static_cast<double>(set.min_p);
    const bool by_k = set.k < a.vocab, by_p = set.p < 1.f;
    const float low = at_least.low;
    if (t == 0) s.i1 = s.i2 = 0;
    __syncthreads();
    for (int i0 = t; i0 < n_runs; i0 += 8 * kThreads) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = rm[min(i0 + e * kThreads, n_runs - 1)];
        uint32_t in = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) in |= static_cast<uint32_t>(i0 + e * kThreads < n_runs && v[e] >= low) << e;
        int at = append(&s.i1, in);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (in >> e & 1) {
                if (at < kSparseRuns) s.runs[at] = i0 + e * kThreads;
                ++at;
            }
    }
    __syncthreads();
    const int runs = s.i1;
    if (runs > kSparseRuns) return false;
    constexpr int kAhead = 16 / L::V;
    for (int i0 = t; i0 < runs * L::kPieces; i0 += kAhead * kThreads) {
        float x[kAhead][L::V];
        int first[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int i = min(i0 + q * kThreads, runs * L::kPieces - 1);
            first[q] = L::token_of_run(s.runs[i / L::kPieces], i % L::kPieces);
            row.x.piece(first[q], x[q]);
        }
        uint32_t in = 0;
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
#pragma unroll
            for (int e = 0; e < L::V; ++e)
                in |= static_cast<uint32_t>(i0 + q * kThreads < runs * L::kPieces && x[q][e] >= low) << (q * L::V + e);
        // (few of a lane's 16, picked one at a time)
        for (int at = append(&s.i2, in); in != 0; in &= in - 1, ++at) {
            const int b = __builtin_ctz(in);
            float v = 0.f;
            int from = 0;
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int e = 0; e < L::V; ++e)
                    if (b == q * L::V + e) v = x[q][e], from = first[q] + e;
            if (at < kList) s.list[at] = number_of(v, from);
        }
    }
    __syncthreads();
    const int n = s.i2;
    if (n > kList) return false;
    sort_down(s.list, n);
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
        if (!by_k && !at_least.min_p && s.cdf[n - 1] < target) return false;
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
        int end = INT32_MIN;  // (negated: the first below the bound)
#pragma unroll
        for (int e = 0; e < per; ++e) {
            const int i = per * t + e;
            if (i > 0 && i < n && w[e] < bound) end = max(end, -i);
        }
        end = wave_max(end);
        if ((t & 63) == 0 && end > INT32_MIN) atomicMin(&s.i0, -end);
        __syncthreads();
        keep = s.i0;
    }
    // the kept tokens in token order, their prefixes, the draws' places among them
    for (int i = t; i < keep; i += kThreads) {
        const uint64_t x = s.list[i];  // (complemented index above the logit's key)
        s.list[i] = (x & ((1 << kIdxBits) - 1)) << 32 | x >> kIdxBits;
    }
    sort_down(s.list, keep);
#pragma unroll
    for (int e = 0; e < per; ++e) {
        const int i = per * t + e;
        sum[e] = i < keep ? row.weight(logit_of(s.list[i] << kIdxBits)) : 0.;
        if (i < kList / 2) s.hits[i] = 0;
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
        atomicAdd(&s.hits[b / 2], 1u << (16 * (b & 1)));
    }
    __syncthreads();
    const auto hits = [&](int i) { return static_cast<int32_t>(s.hits[i / 2] >> (16 * (i & 1)) & 0xffff); };
    uint32_t mine = 0, groups;
#pragma unroll
    for (int e = 0; e < per; ++e) mine += hits(per * t + e) > 0;
    uint32_t at = block_scan(mine, reinterpret_cast<uint32_t*>(s.part), groups);
#pragma unroll
    for (int e = 0; e < per; ++e) {
        const int i = per * t + e;
        if (hits(i) > 0) {
            a.token[set.off + at] = (1 << kIdxBits) - 1 - static_cast<int32_t>(s.list[i] >> 32);
            a.count[set.off + at] = hits(i);
            ++at;
        }
    }
    if (t == 0) a.n_groups[r] = static_cast<int32_t>(groups);
    return true;
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(6))) void filter_draw(Args a) {
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
    const double* ps = a.part_sum + static_cast<int64_t>(r) * a.tiles * L::kPieces;

    // the largest logit, the smallest for the bins below, and the tiles' weights relative to the row's largest
    const bool by_k = set.k < a.vocab, by_p = set.p < 1.f;
    const float* sample = a.sample + static_cast<int64_t>(r) * a.tiles * 128;
    const float2* tm = a.tile_max + static_cast<int64_t>(r) * a.tiles;
    float top = -INFINITY, low = INFINITY;
    for (int i = t; i < a.tiles; i += kThreads) {
        const float2 v = tm[i];
        top = fmaxf(top, v.x), low = fminf(low, v.y);
    }
    top = wave_max(top), low = -wave_max(-low);
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
        for (int i = t; i < a.tiles; i += kThreads) {
            double sum = 0.;
#pragma unroll
            for (int j = 0; j < L::kPieces; ++j) sum += ps[i * L::kPieces + j];
            s.tile[i + 1] = sum * row.weight(tm[i].x);
        }
        tile_prefixes(s, a.tiles);
        whole = s.tile[a.tiles];
        if (!by_p) {
            draw_from_tiles<BF16>(
                s, a, r, row, set, [&](int tile, int j) { return ps[tile * L::kPieces + j] * row.weight(tm[tile].x); },
                [&](int, float v) { return row.weight(v); });
            return;
        }
        __syncthreads();
    }
    // bins wide enough for what can be drawn
    const float width = set.temp > 0.f ? fminf(top - low, 100.f * set.temp) : top - low;
    const float scale = width > 0.f ? fminf((kHist - 1) / width, 1e30f) : 0.f;
    const double bound = static_cast<double>(set.min_p);
    // min-p alone, or before top-p, if few runs reach it
    Bound at_least{0.f, true, kHist, -1, 0};
    if (!by_k && bound > 0.) {
        // (by a little, and to the next float below)
        const double foot = row.top + (log2(bound) - 1e-6) / row.c;
        at_least.low = foot > -3.4e38 ? __double2float_rd(foot) : -3.4028234663852886e38f;
        if (t == 0) s.i0 = 0;
        __syncthreads();
        int mine = 0;
        each_of(rm, a.tiles * 64, [&](int, float v) { mine += v >= at_least.low; });
        if (mine) atomicAdd(&s.i0, mine);
        __syncthreads();
        at_least.runs = s.i0;
        __syncthreads();
        if (at_least.runs <= kSparseFew) {
            if (draw_from_runs<BF16>(s, a, r, row, set, rm, whole, at_least)) return;
            __syncthreads();  // every wave has read the count that made it fail
        }
    }
    if (by_k || by_p) {
        at_least = find_bound<BF16>(s, a, row, set, rm, sample, top, scale, whole);
        if (at_least.runs <= kSparseRuns && draw_from_runs<BF16>(s, a, r, row, set, rm, whole, at_least)) return;
    }
    if (t == 0) {
        Again again{};
        again.row = r;
        again.whole_row = a.cap == 0 || (by_k && set.k > a.cap);
        again.first = at_least.first, again.last = at_least.last;
        again.top = top, again.scale = scale, again.weight = whole;
        a.again[atomicAdd(a.n_again, 1)] = again;
    }
}

// A wave a tile of the rows that are read again: the weight above the interval, of what min-p keeps of it, and the
// numbers inside.
template <bool BF16>
__global__ __launch_bounds__(kScanThreads) void filter_narrow(Args a) {
    using L = Logits<BF16>;
    const int lane = threadIdx.x & 63;
    const int64_t items = static_cast<int64_t>(*a.n_again) * a.tiles;
    const int waves = gridDim.x * (kScanThreads / 64);
    for (int64_t id = blockIdx.x * (kScanThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); id < items; id += waves) {
        const int d = static_cast<int>(id / a.tiles), tile = static_cast<int>(id - static_cast<int64_t>(d) * a.tiles);
        const Again g = a.again[d];
        if (g.whole_row) continue;
        const Settings set = settings_of(a, g.row);
        const Row<BF16> row{{static_cast<const char*>(a.logits) + g.row * a.stride * (BF16 ? 2 : 4), a.vocab},
                            static_cast<double>(g.top), set.scale()};
        const double bound = static_cast<double>(set.min_p);
        float x[L::kPieces][L::V];
        row.x.tile(tile * kTile, lane, x);
        double above = 0., kept[L::kPieces];
        uint32_t in = 0;
#pragma unroll
        for (int j = 0; j < L::kPieces; ++j) {
            kept[j] = 0.;
#pragma unroll
            for (int e = 0; e < L::V; ++e) {
                const int b = bin_of(x[j][e], g.top, g.scale);
                if (b < g.first) {
                    const double y = row.weight(x[j][e]);
                    above += y;
                    kept[j] += y >= bound ? y : 0.;
                } else if (b <= g.last && x[j][e] > -INFINITY) {
                    in |= 1u << (j * L::V + e);
                }
            }
        }
        above = lane_of(wave_scan(above), 63);
        const double part = wave_sums(kept, lane);
        const int64_t at = static_cast<int64_t>(g.row) * a.tiles + tile;
        if (lane == 0) a.above[at] = above;
        if (lane % (64 / L::kPieces) == 0) a.kept[at * L::kPieces + lane / (64 / L::kPieces)] = part;
        int base = append(&a.again[d].n, in);
        // (few of a lane's 32, read again from the cache: 38 us of 129 rows of 151,936, 45 us picked out of the registers)
        uint64_t* list = a.lists + static_cast<int64_t>(g.row) * a.cap;
        for (; in != 0; in &= in - 1, ++base) {
            const int q = __builtin_ctz(in), i = L::token(tile * kTile, lane, q / L::V) + q % L::V;
            if (base < a.cap) list[base] = number_of(row.x.at(i), i);
        }
    }
}

// The kept weight of a row's parts, read whole by the workgroup.
template <bool BF16, class F>
__device__ __forceinline__ void sum_parts(const Args& a, const Row<BF16>& row, double* parts, F kept) {
    using L = Logits<BF16>;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int i = w; i < a.tiles; i += kWaves) {
        float x[L::kPieces][L::V];
        row.x.tile(i * kTile, lane, x);
        double sum[L::kPieces];
#pragma unroll
        for (int j = 0; j < L::kPieces; ++j) {
            sum[j] = 0.;
#pragma unroll
            for (int e = 0; e < L::V; ++e) sum[j] += kept(L::token(i * kTile, lane, j) + e, x[j][e]);
        }
        const double part = wave_sums(sum, lane);
        if (lane % (64 / L::kPieces) == 0) parts[i * L::kPieces + lane / (64 / L::kPieces)] = part;
    }
}

// The threshold of a row that filter_narrow has read, and the kept weight of its list in each part (`inside`, zero
// before); false if the threshold is not in the list.
template <bool BF16>
__device__ bool cut_in_list(Shared& s, const Args& a, const Row<BF16>& row, const Settings& set, const Again& g, uint64_t* inside,
                            uint64_t& cut) {
    const int t = threadIdx.x;
    const int64_t at = static_cast<int64_t>(g.row) * a.tiles;
    const double bound = static_cast<double>(set.min_p);
    cut = 0;
    const bool by_k = set.k < a.vocab;
    if (by_k || set.p < 1.f) {
        if (g.n > a.cap || (by_k && g.n < set.k && g.last < kHist - 1)) return false;
        static_assert(kMine * kThreads >= 8192, "a list of any length");
        const uint64_t* from = a.lists + static_cast<int64_t>(g.row) * a.cap;
        ListNumbers list;
#pragma unroll
        for (int e = 0; e < kMine; ++e) list.n[e] = t + e * kThreads < g.n ? from[t + e * kThreads] : 0;
        double sum = 0., above;
        for (int i = t; i < a.tiles; i += kThreads) sum += a.above[at + i];
        block_scan(sum, s.partd, above);
        const double want = static_cast<double>(set.p) * g.weight - above;
        // the list's weight in units, and its smallest and largest number
        uint64_t units = 0, all, lo = ~uint64_t{0}, hi = 0;
#pragma unroll
        for (int e = 0; e < kMine; ++e) {
            list.w[e] = 0;
            if (t + e * kThreads < g.n) {
                units += list.w[e] = row.units(logit_of(list.n[e]));
                lo = list.n[e] < lo ? list.n[e] : lo, hi = list.n[e] > hi ? list.n[e] : hi;
            }
        }
        block_scan(units, s.part, all);
        if (!by_k && (!(want > 0.) || static_cast<double>(all) < want * kUnit)) return false;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const uint64_t l2 = __shfl_xor(lo, o), h2 = __shfl_xor(hi, o);
            lo = l2 < lo ? l2 : lo, hi = h2 > hi ? h2 : hi;
        }
        __syncthreads();
        if (t == 0) s.u0 = ~uint64_t{0}, s.u1 = 0;
        __syncthreads();
        if ((t & 63) == 0) {
            atomicMin(reinterpret_cast<unsigned long long*>(&s.u0), static_cast<unsigned long long>(lo));
            atomicMax(reinterpret_cast<unsigned long long*>(&s.u1), static_cast<unsigned long long>(hi));
        }
        __syncthreads();
        lo = s.u0, hi = s.u1;
        const auto units_of = [&](float v) { return row.units(v); };
        // the k-th, then the end of top-p from there up
        cut = lo;
#pragma unroll 1
        for (int by_mass = by_k ? 0 : 1; by_mass <= (set.p < 1.f ? 1 : 0); ++by_mass)
            cut = find_cut(s, list, units_of, by_mass != 0, by_k, cut, hi, static_cast<uint64_t>(set.k), by_k ? static_cast<double>(set.p) : want * kUnit);
        // kept tokens of the list, by part: integers, whatever their order
        list.each([&](uint64_t n, uint64_t) {
            if (n < cut) return;
            const double y = row.weight(logit_of(n));
            if (y < bound) return;
            const int i = (1 << kIdxBits) - 1 - static_cast<int>(n & ((1 << kIdxBits) - 1));
            atomicAdd(reinterpret_cast<unsigned long long*>(&inside[i / (64 * Logits<BF16>::V)]), static_cast<unsigned long long>(y * kFine + .5));
        });
    }
    return true;
}

// Cuts and draws of the rows that are read again, a workgroup a row.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void filter_finish(Args a) {
    using L = Logits<BF16>;
    __shared__ Shared s;
    __shared__ uint64_t inside[kMaxTiles * L::kPieces];
    const int t = threadIdx.x;
    for (int d = blockIdx.x; d < *a.n_again; d += gridDim.x) {
        __syncthreads();
        for (int i = t; i < a.tiles * L::kPieces; i += kThreads) inside[i] = 0;
        const Again g = a.again[d];
        const Settings set = settings_of(a, g.row);
        const Row<BF16> row{{static_cast<const char*>(a.logits) + g.row * a.stride * (BF16 ? 2 : 4), a.vocab},
                            static_cast<double>(g.top), set.scale()};
        const double bound = static_cast<double>(set.min_p);
        double* parts = a.kept + static_cast<int64_t>(g.row) * a.tiles * L::kPieces;
        uint64_t cut = 0;
        auto kept = [&](int i, float v) {
            const double x = row.weight(v);
            return number_of(v, i) >= cut && x >= bound ? x : 0.;
        };
        bool sums = g.whole_row || !cut_in_list<BF16>(s, a, row, set, g, inside, cut);
        if (!sums) {
            // `inside` misses weights below 2^-51, up to 2^-38 together: draws that fall so low (one in 2^30) take the parts'
            // own sums instead
            int low = 0;
            for (int i = t; i < set.n; i += kThreads) low |= a.uniform[set.off + i] < 0x1p-30f;
            sums = __syncthreads_or(low);
            if (sums)
                for (int i = t; i < a.tiles * L::kPieces; i += kThreads) inside[i] = 0;
        } else {
            const RowNumbers<BF16> all{row.x};
            auto units = [&](float v) { return row.units(v); };
            const uint64_t lo = static_cast<uint64_t>(key_of(-3.4028234663852886e38f)) << kIdxBits;
            const uint64_t hi = number_of(g.top, 0);
            cut = lo;
            if (set.k >= a.vocab && set.p >= 1.f) cut = 0;
#pragma unroll 1
            for (int by_mass = set.k < a.vocab ? 0 : 1; by_mass <= (set.p < 1.f ? 1 : 0); ++by_mass)
                cut = find_cut(s, all, units, by_mass != 0, true, cut, hi, static_cast<uint64_t>(set.k), static_cast<double>(set.p));
        }
        if (sums) sum_parts<BF16>(a, row, parts, kept);
        __syncthreads();
        const auto part = [&](int tile, int j) {
            return parts[tile * L::kPieces + j] + static_cast<double>(inside[tile * L::kPieces + j]) / kFine;
        };
        for (int i = t; i < a.tiles; i += kThreads) {
            double sum = 0.;
#pragma unroll
            for (int j = 0; j < L::kPieces; ++j) sum += part(i, j);
            s.tile[i + 1] = sum;
        }
        tile_prefixes(s, a.tiles);
        draw_from_tiles<BF16>(s, a, g.row, row, set, part, kept);
    }
}

}  // namespace

int tkv::launch_filter_sample(const FilterCall& f, void* stream) {
    Args a{};
    a.n_rows = f.n_rows, a.vocab = f.vocab, a.logits = f.logits, a.stride = f.stride;
    a.temperature = f.temperature, a.top_k = f.top_k, a.top_p = f.top_p, a.min_p = f.min_p;
    a.uniform = f.uniform, a.draw_off = f.draw_off, a.n_draws = f.n_draws;
    a.token = f.token, a.count = f.count, a.n_groups = f.n_groups;
    const FilterLayout l = filter_layout(f.n_rows, f.vocab);
    uint8_t* ws = static_cast<uint8_t*>(f.workspace);
    a.tiles = l.tiles, a.cap = l.list;
    a.n_again = reinterpret_cast<int32_t*>(ws);
    a.again = reinterpret_cast<Again*>(ws + l.rows);
    a.part_sum = reinterpret_cast<double*>(ws + l.part_sum);
    a.above = reinterpret_cast<double*>(ws + l.above);
    a.kept = reinterpret_cast<double*>(ws + l.kept);
    a.tile_max = reinterpret_cast<float2*>(ws + l.tile_max);
    a.run_max = reinterpret_cast<float*>(ws + l.run_max);
    a.sample = reinterpret_cast<float*>(ws + l.sample);
    a.lists = reinterpret_cast<uint64_t*>(ws + l.lists);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    constexpr int waves = kScanThreads / 64;
    const int64_t grid = (static_cast<int64_t>(f.n_rows) * a.tiles + waves - 1) / waves;
    // (a launch takes less than 2^32 threads)
    if (grid * kScanThreads > UINT32_MAX || static_cast<int64_t>(f.n_rows) * kThreads > UINT32_MAX)
        return set_error(TKV_EINVAL, "tkv_filter_sample: %d rows are too many", f.n_rows);
    const auto launch = [&](auto scan, auto draw, auto narrow, auto finish) {
        scan<<<dim3(static_cast<unsigned>(grid)), dim3(kScanThreads), 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;  // (the others read what it writes)
        draw<<<dim3(static_cast<unsigned>(f.n_rows)), dim3(kThreads), 0, st>>>(a);
        narrow<<<dim3(static_cast<unsigned>(std::min<int64_t>(grid, 2048))), dim3(kScanThreads), 0, st>>>(a);
        finish<<<dim3(static_cast<unsigned>(std::min(f.n_rows, 1024))), dim3(kThreads), 0, st>>>(a);
        return hipGetLastError();
    };
    const bool past = static_cast<int64_t>(f.n_rows) * f.vocab * (f.logit_type == TKV_LOGITS_BF16 ? 2 : 4) >= int64_t{192} << 20;
    const hipError_t e =
        f.logit_type == TKV_LOGITS_BF16
            ? launch(past ? filter_scan<true, true> : filter_scan<true, false>, filter_draw<true>, filter_narrow<true>, filter_finish<true>)
            : launch(past ? filter_scan<false, true> : filter_scan<false, false>, filter_draw<false>, filter_narrow<false>, filter_finish<false>);
    return e == hipSuccess ? TKV_OK : set_error(TKV_EHIP, "tkv_filter_sample launch: %s", hipGetErrorString(e));
}
