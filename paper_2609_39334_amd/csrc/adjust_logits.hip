// Logits under the rules of their rows (tkv_adjust_logits): penalties for the tokens of each row's path, biases, a grammar's
// mask.  The path's tokens lie in a paged pool of their own, under the same kind of tables as its keys.
//
// A workgroup takes a tile of consecutive tokens of the vocabulary for a few query tokens of one row.  It counts in LDS how
// often each of them occurs in the row's context, adds the drafted tokens that a query token sees (and takes them out again
// before the next one), and passes once over the tile's logits.  Counts are whole numbers, so the order in which threads add
// them changes nothing.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cstdint>

#include "internal.h"
#include "rows.h"

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kTile = 8192;                        // tokens of the vocabulary a workgroup
constexpr int kLoads = kTile / (4 * kThreads);     // four tokens a load
constexpr int kMaxDraft = 1024;
constexpr uint32_t kInPrompt = 0x80000000u, kTimes = 0x7fffffffu;  // a count: seen in the prompt; occurrences past it
constexpr int32_t kPast = 1 << 30;                 // a drafted token past the prompt

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4_t __attribute__((ext_vector_type(4)));
// rows start anywhere
typedef f32x4_t f32x4_u __attribute__((aligned(4)));
typedef u16x4_t u16x4_u __attribute__((aligned(2)));

struct Args {
    tkv_draft_batch b;
    tkv_logit_rules u;
    int32_t num_blocks, vocab, n_tiles, groups, per;  // groups of `per` query tokens of a row
    const int32_t* tokens;
    const void* in;
    void* out;
    int64_t in_stride, out_stride;
};

template <bool B16>
__device__ __forceinline__ f32x4_t load4(const void* row, int c, int n) {
    f32x4_t x{0.f, 0.f, 0.f, 0.f};
    if constexpr (B16) {
        const uint16_t* p = static_cast<const uint16_t*>(row) + c;
        u16x4_t v{0, 0, 0, 0};
        if (c + 4 <= n)
            v = *reinterpret_cast<const u16x4_u*>(p);
        else
            for (int e = 0; e < 3; ++e)
                if (c + e < n) v[e] = p[e];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(static_cast<uint32_t>(v[e]) << 16);
    } else {
        const float* p = static_cast<const float*>(row) + c;
        if (c + 4 <= n)
            x = *reinterpret_cast<const f32x4_u*>(p);
        else
            for (int e = 0; e < 3; ++e)
                if (c + e < n) x[e] = p[e];
    }
    return x;
}

template <bool B16>
__device__ __forceinline__ void store4(void* row, int c, int n, f32x4_t x) {
    if constexpr (B16) {
        uint16_t* p = static_cast<uint16_t*>(row) + c;
        const u16x4_t v = __builtin_bit_cast(u16x4_t, __builtin_convertvector(x, bf16x4_t));
        if (c + 4 <= n)
            *reinterpret_cast<u16x4_u*>(p) = v;
        else
            for (int e = 0; e < 3; ++e)
                if (c + e < n) p[e] = v[e];
    } else {
        float* p = static_cast<float*>(row) + c;
        if (c + 4 <= n)
            *reinterpret_cast<f32x4_u*>(p) = x;
        else
            for (int e = 0; e < 3; ++e)
                if (c + e < n) p[e] = x[e];
    }
}

template <bool IN16, bool OUT16, bool BIAS>
__global__ __launch_bounds__(kThreads) void adjust(Args a) {
    __shared__ __attribute__((aligned(16))) uint32_t count[kTile];
    __shared__ __attribute__((aligned(16))) int32_t given[BIAS ? kTile : 4];  // a token's last bias, as its number + 1
    __shared__ int32_t drafted[kMaxDraft];  // a drafted token's place in the tile, with kPast; -1: not in it
    __shared__ int part[2][kWaves];
    const int tid = threadIdx.x;
    const int tile = blockIdx.x % a.n_tiles, g = blockIdx.x / a.n_tiles;
    const int r = g / a.groups;
    const tkv::RowTokens t = tkv::row_tokens(a.b, r);
    const int first = (g - r * a.groups) * a.per;
    if (!t.ok || first >= t.L) return;
    const int end = min(t.L, first + a.per);
    const int c0 = tile * kTile, n = min(kTile, a.vocab - c0);
    const char* in = static_cast<const char*>(a.in) + (static_cast<int64_t>(t.q0 + first) * a.in_stride + c0) * (IN16 ? 2 : 4);
    char* out = static_cast<char*>(a.out) + (static_cast<int64_t>(t.q0 + first) * a.out_stride + c0) * (OUT16 ? 2 : 4);
    const int64_t in_step = a.in_stride * (IN16 ? 2 : 4), out_step = a.out_stride * (OUT16 ? 2 : 4);

    f32x4_t x[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) x[k] = load4<IN16>(in, (k * kThreads + tid) * 4, n);

    const tkv::RowTable tab = tkv::row_table(a.b.kv_indptr, r, a.b.n_kv_blocks, a.b.max_blocks);
    const float rep = a.u.repetition ? a.u.repetition[r] : 1.f;
    const float pres = a.u.presence ? a.u.presence[r] : 0.f;
    const float freq = a.u.frequency ? a.u.frequency[r] : 0.f;
    const int prompt = a.u.prompt_len ? a.u.prompt_len[r] : 0;
    tkv::RowTable bias{0, 0, true};
    if (BIAS) bias = tkv::row_table(a.u.bias_indptr, r, a.u.n_bias, a.u.n_bias);
    const bool ok = tab.ok && bias.ok && rep > 0.f && rep < INFINITY && fabsf(pres) < INFINITY && fabsf(freq) < INFINITY;
    const bool counts = ok && (rep != 1.f || pres != 0.f || freq != 0.f);
    const bool biased = BIAS && ok && bias.n > 0;

    if (counts) {
        for (int c = tid * 4; c < kTile; c += kThreads * 4) *reinterpret_cast<uint4*>(count + c) = uint4{0, 0, 0, 0};
        for (int j = tid; j < t.L; j += kThreads) drafted[j] = -1;
    }
    if (biased)
        for (int c = tid * 4; c < kTile; c += kThreads * 4) *reinterpret_cast<uint4*>(given + c) = uint4{0, 0, 0, 0};
    if (counts || biased) __syncthreads();
    if (biased) {
        for (int e = tid; e < bias.n; e += kThreads) {
            const uint32_t at = static_cast<uint32_t>(a.u.bias_token[bias.first + e]) - static_cast<uint32_t>(c0);
            if (at < static_cast<uint32_t>(n)) atomicMax(given + at, e + 1);
        }
    }
    if (counts) {
        int N = 0;
        if (tab.n > kThreads) {
            int mine = 0, id;
            for (int e = tid; e < tab.n; e += kThreads) mine += tkv::entry_len(a.b.kv_blocks, a.b.block_len, a.num_blocks, tab.first + e, id);
            tkv::group_before<kWaves>(mine, N, part[1]);
        }
        int run = 0;
        for (int base = 0; base < tab.n; base += kThreads) {
            int id = 0, len = 0, total;
            if (base + tid < tab.n) len = tkv::entry_len(a.b.kv_blocks, a.b.block_len, a.num_blocks, tab.first + base + tid, id);
            int4 tok[4];
            if (len > 0) {
                const int4* p = reinterpret_cast<const int4*>(a.tokens + static_cast<int64_t>(id) * tkv::kBlock);
#pragma unroll
                for (int q = 0; q < 4; ++q) tok[q] = p[q];
            }
            const int before = run + tkv::group_before<kWaves>(len, total, part[0]);
            if (tab.n <= kThreads) N = total;
            run += total;
            const int context = N - t.L;
            if (len > 0) {
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const uint32_t at = static_cast<uint32_t>((&tok[0].x)[q]) - static_cast<uint32_t>(c0);
                    if (q >= len || at >= static_cast<uint32_t>(n)) continue;
                    const int number = before + q;
                    if (number >= context)
                        drafted[number - context] = static_cast<int32_t>(at) | (number >= prompt ? kPast : 0);
                    else if (number >= prompt)
                        atomicAdd(count + at, 1u);
                    else
                        atomicOr(count + at, kInPrompt);
                }
            }
            __syncthreads();  // (part is free again; after the last round: everything is counted)
        }
    }
    if (biased) __syncthreads();

    const float inv = 1.f / rep;
    for (int i = first; i < end; ++i) {
        const int64_t q = t.q0 + i;
        uint32_t put = 0;  // which of this thread's drafted tokens were the first to be seen in the prompt
        if (counts) {
            const uint64_t* mask = a.b.mask + q * a.b.mask_words;
            int b = 0;
            for (int j = tid; j < t.L; j += kThreads, ++b) {
                const int32_t d = drafted[j];
                if (d < 0 || !(mask[j >> 6] >> (j & 63) & 1)) continue;
                if (d & kPast)
                    atomicAdd(count + (d & ~kPast), 1u);
                else if (!(atomicOr(count + d, kInPrompt) & kInPrompt))
                    put |= 1u << b;
            }
            __syncthreads();
        }
        const int grammar = a.u.grammar ? a.u.grammar[q] : -1;
        const bool fine = ok && grammar < a.u.n_grammars;
        const uint32_t* allowed = grammar >= 0 && fine ? a.u.allowed + static_cast<int64_t>(grammar) * a.u.allowed_words : nullptr;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int c = (k * kThreads + tid) * 4;
            if (c >= n) continue;
            f32x4_t y = x[k];
            if (counts) {
                const uint4 s4 = *reinterpret_cast<const uint4*>(count + c);
                const uint32_t* s = &s4.x;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (s[e] != 0) y[e] = y[e] > 0.f ? y[e] * inv : y[e] * rep;
                    const uint32_t times = s[e] & kTimes;
                    if (times != 0) y[e] = y[e] - freq * static_cast<float>(times) - pres;
                }
            }
            if (biased) {
                const int4 w4 = *reinterpret_cast<const int4*>(given + c);
                const int32_t* w = &w4.x;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (w[e] != 0) y[e] += a.u.bias_value[bias.first + w[e] - 1];
            }
            if (allowed) {
                const uint32_t bits = allowed[(c0 + c) >> 5] >> ((c0 + c) & 31);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!(bits >> e & 1)) y[e] = -INFINITY;
            }
            if (!fine) y = f32x4_t{NAN, NAN, NAN, NAN};
            store4<OUT16>(out, c, n, y);
        }
        in += in_step, out += out_step;
        if (i + 1 == end) break;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) x[k] = load4<IN16>(in, (k * kThreads + tid) * 4, n);
        if (counts) {
            __syncthreads();
            int b = 0;
            const uint64_t* mask = a.b.mask + q * a.b.mask_words;
            for (int j = tid; j < t.L; j += kThreads, ++b) {
                const int32_t d = drafted[j];
                if (d < 0 || !(mask[j >> 6] >> (j & 63) & 1)) continue;
                if (d & kPast)
                    atomicSub(count + (d & ~kPast), 1u);
                else if (put >> b & 1)
                    atomicAnd(count + d, kTimes);
            }
            __syncthreads();
        }
    }
}

}  // namespace

int tkv::launch_adjust_logits(const AdjustCall& f, void* stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    Args a{};
    a.b = f.b, a.u = f.u;
    a.num_blocks = f.num_blocks, a.vocab = f.vocab, a.tokens = f.tokens;
    a.in = f.in, a.out = f.out, a.in_stride = f.in_stride, a.out_stride = f.out_stride;
    a.n_tiles = (f.vocab + kTile - 1) / kTile;
    const int64_t units = static_cast<int64_t>(a.n_tiles) * f.b.n_qtok;
    a.per = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(8, f.b.max_q), units / 2048)));
    a.groups = (f.b.max_q + a.per - 1) / a.per;
    const int64_t grid = static_cast<int64_t>(a.n_tiles) * a.groups * f.b.n_rows;
    if (grid > INT32_MAX)
        return set_error(TKV_EINVAL, "tkv_adjust_logits: %lld workgroups are too many", static_cast<long long>(grid));
    const auto run = [&](auto kernel) { kernel<<<dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, st>>>(a); };
    const bool bias = f.u.n_bias > 0;
    if (f.in16)
        f.out16 ? (bias ? run(adjust<true, true, true>) : run(adjust<true, true, false>))
                : (bias ? run(adjust<true, false, true>) : run(adjust<true, false, false>));
    else
        f.out16 ? (bias ? run(adjust<false, true, true>) : run(adjust<false, true, false>))
                : (bias ? run(adjust<false, false, true>) : run(adjust<false, false, false>));
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TKV_OK : set_error(TKV_EHIP, "tkv_adjust_logits launch: %s", hipGetErrorString(e));
}
