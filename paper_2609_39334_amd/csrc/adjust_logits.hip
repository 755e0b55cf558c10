// Logits under the rules of their rows (tkv_adjust_logits): penalties for the tokens of each row's path, biases, a grammar's
// mask.  The path's tokens lie in a paged pool of their own, under the same kind of tables as its keys.
//
// A workgroup takes a tile of consecutive tokens of the vocabulary for a few query tokens of one row.  It counts in LDS how
// often each of them occurs in the row's context, adds the drafted tokens that a query token sees (and takes them out again
// before the next one), and passes once over the tile's logits.  Counts are whole numbers, so the order in which threads add
// them changes nothing.
//
// Logits are read and written once and that bounds large calls: 1,000 rows of 151,936 in fp32 take 228 us, 5.35 TB/s, a large
// copy's rate.  Every tile walks its row's path (4 bytes a token, from L2 after the first), which bounds few rows: five of
// 151,936, bf16, paths of 200 to 1,000 tokens 9 us; 16 rows with paths of 8,000 to 30,000 tokens 16 us, about four entries of a
// table a thread, eleven instructions a token (by 25, 18); 16 trees of 4 to 32 tokens, 32,003, bf16 to fp32, 19 us: the row, its
// table, lengths, tokens and counts are a chain, before which the logits are asked for.
//
// Measured for the choices below (threads / tile, before logits went past the caches): 256 / 8,192 with many tiles, the 1,000 rows
// 239 to 249 us; 512 / 8,192 250; 256 / 4,096 261; 512 / 16,384 246; 1,024 / 8,192 446; 1,024 / 16,384 310.  512 / 8,192 with few:
// the five rows 8.7 us, by 256 11.0; the paths of 30,000 tokens 18 and 26.  (256 rows with paths of 8,000 to 16,000 tokens: 143 by
// 512, 120 by 256.)
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "internal.h"
#include "rows.h"

namespace {

constexpr int kTile = 8192;                        // tokens of the vocabulary a workgroup
constexpr int kMaxDraft = 1024;
// Logits of many rows do not stay in the caches until they are drawn from.  Written past them from 8 MiB on: 238 bf16 rows of
// 32,003 21.4 us, 22.8 into them (45.5 and 46.5 with the draws after them); five of 151,936 cost a draw 0.9 us more.  Read
// past them where both pass 192 MiB: 1,000 fp32 rows of 151,936 234 us, 244 with the stores alone, 252 through the caches.
constexpr int64_t kPastOut = 8 << 20, kPastIn = 192 << 20;
constexpr int kBatch = 4;                          // entries of a table a thread looks at together
constexpr int32_t kPast = 1 << 30;                 // a drafted token past the prompt

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4_t __attribute__((ext_vector_type(4)));
// rows start anywhere
typedef f32x4_t f32x4_u __attribute__((aligned(4)));
typedef u16x4_t u16x4_u __attribute__((aligned(2)));

struct Args {
    tkv_draft_batch b;
    tkv_logit_rules u;
    int32_t num_blocks, vocab, n_tiles, groups, per, units;  // groups of `per` query tokens of a row; groups or tokens in all
    bool spread, search;
    bool past_in, past_out;  // logits read and written past the caches
    const int32_t* tokens;
    const void* in;
    void* out;
    int64_t in_stride, out_stride;
};

// PAST: past the caches.
template <bool B16, bool PAST>
__device__ __forceinline__ f32x4_t load4(const void* row, int c, int n) {
    const auto get = [](const auto* p) {
        if constexpr (PAST) return __builtin_nontemporal_load(p);
        else return *p;
    };
    f32x4_t x{0.f, 0.f, 0.f, 0.f};
    if constexpr (B16) {
        const uint16_t* p = static_cast<const uint16_t*>(row) + c;
        u16x4_t v{0, 0, 0, 0};
        if (c + 4 <= n)
            v = get(reinterpret_cast<const u16x4_u*>(p));
        else
            for (int e = 0; e < 3; ++e)
                if (c + e < n) v[e] = p[e];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(static_cast<uint32_t>(v[e]) << 16);
    } else {
        const float* p = static_cast<const float*>(row) + c;
        if (c + 4 <= n)
            x = get(reinterpret_cast<const f32x4_u*>(p));
        else
            for (int e = 0; e < 3; ++e)
                if (c + e < n) x[e] = p[e];
    }
    return x;
}

template <bool B16>
__device__ __forceinline__ void store4(void* row, int c, int n, f32x4_t x, bool past) {
    const auto set = [past](auto* p, auto v) {
        if (past) {
            asm volatile("");  // (the branches would be made one, and the store an ordinary one)
            __builtin_nontemporal_store(v, p);
            asm volatile("");
        } else {
            *p = v;
        }
    };
    if constexpr (B16) {
        uint16_t* p = static_cast<uint16_t*>(row) + c;
        const u16x4_t v = __builtin_bit_cast(u16x4_t, __builtin_convertvector(x, bf16x4_t));
        if (c + 4 <= n)
            set(reinterpret_cast<u16x4_u*>(p), v);
        else
            for (int e = 0; e < 3; ++e)
                if (c + e < n) p[e] = v[e];
    } else {
        float* p = static_cast<float*>(row) + c;
        if (c + 4 <= n)
            set(reinterpret_cast<f32x4_u*>(p), x);
        else
            for (int e = 0; e < 3; ++e)
                if (c + e < n) p[e] = x[e];
    }
}

// What a tile's tokens have of something, a number of 16 bits each (two in a word of LDS) or of 32.
template <bool WIDE>
struct Cells {
    using Four = std::conditional_t<WIDE, uint4, uint2>;
    static constexpr int kWords = WIDE ? kTile : kTile / 2;
    static constexpr uint32_t kPrompt = WIDE ? 0x80000000u : 0x8000u, kTimes = kPrompt - 1;  // seen in the prompt; times past it
    uint32_t* at;
    static __device__ __forceinline__ int shift(uint32_t i) { return WIDE ? 0 : i << 4 & 31; }
    __device__ __forceinline__ uint32_t* word(uint32_t i) const { return at + (WIDE ? i : i >> 1); }
    __device__ __forceinline__ void clear(int tid, int threads) const {
        for (int i = tid * 4; i < kWords; i += threads * 4) *reinterpret_cast<uint4*>(at + i) = uint4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void more(uint32_t i) const { atomicAdd(word(i), 1u << shift(i)); }
    __device__ __forceinline__ void less(uint32_t i) const { atomicSub(word(i), 1u << shift(i)); }
    __device__ __forceinline__ void set(uint32_t i) const { atomicOr(word(i), kPrompt << shift(i)); }
    __device__ __forceinline__ bool mark(uint32_t i) const {  // whether it was not marked before
        return !(atomicOr(word(i), kPrompt << shift(i)) >> shift(i) & kPrompt);
    }
    __device__ __forceinline__ void unmark(uint32_t i) const { atomicAnd(word(i), ~(kPrompt << shift(i))); }
    __device__ __forceinline__ void raise(uint32_t i, uint32_t to) const {  // to the largest of those given
        if (WIDE) {
            atomicMax(word(i), to);
            return;
        }
        uint32_t old = *word(i);
        while ((old >> shift(i) & 0xffff) < to) {
            const uint32_t seen = atomicCAS(word(i), old, (old & ~(0xffffu << shift(i))) | to << shift(i));
            if (seen == old) break;
            old = seen;
        }
    }
    __device__ __forceinline__ void four(int i, uint32_t (&x)[4]) const {
        const Four f = *reinterpret_cast<const Four*>(word(i));
        if constexpr (WIDE)
            x[0] = f.x, x[1] = f.y, x[2] = f.z, x[3] = f.w;
        else
            x[0] = f.x & 0xffff, x[1] = f.x >> 16, x[2] = f.y & 0xffff, x[3] = f.y >> 16;
    }
};

template <bool IN16, bool OUT16, bool BIAS, bool WIDE, int kThreads>
__global__ __launch_bounds__(kThreads) void adjust(Args a) {
    using Cell = Cells<WIDE>;
    constexpr int kWaves = kThreads / 64, kLoads = kTile / (4 * kThreads);  // four tokens a load
    __shared__ __attribute__((aligned(16))) uint32_t counted[Cell::kWords];
    __shared__ __attribute__((aligned(16))) uint32_t biases[BIAS ? Cell::kWords : 4];
    __shared__ int32_t drafted[kMaxDraft];  // a drafted token's place in the tile, with kPast; -1: not in it
    __shared__ int part[kWaves];
    const Cell count{counted}, given{biases};  // given: a token's last bias, as its number + 1
    const int tid = threadIdx.x;
    int tile = blockIdx.x % a.n_tiles, g = blockIdx.x / a.n_tiles;
    if (a.spread) {  // a row's tiles on one XCD, whose L2 then holds its path
        const int of8 = blockIdx.x >> 3;
        tile = of8 % a.n_tiles, g = of8 / a.n_tiles * 8 + (blockIdx.x & 7);
        if (g >= a.units) return;
    }
    // what the row is: all of it is asked for before anything is waited for
    int r = g % a.b.n_rows;
    if (a.search) {  // g is a query token: its row
        __shared__ int row;
        if (tid == 0) row = INT32_MAX;
        __syncthreads();
        for (int r0 = 0; r0 < a.b.n_rows; r0 += kThreads) {
            const int mine = r0 + tid;
            const tkv::RowTokens m = mine < a.b.n_rows ? tkv::row_tokens(a.b, mine) : tkv::RowTokens{};
            if (m.ok && g >= m.q0 && g < m.q0 + m.L) atomicMin(&row, mine);
            if (__syncthreads_or(m.ok && g >= m.q0 && g < m.q0 + m.L)) break;
        }
        r = __builtin_amdgcn_readfirstlane(row);
        if (r == INT32_MAX) return;
    }
    const tkv::RowTokens t = tkv::row_tokens(a.b, r);
    const tkv::RowTable tab = tkv::row_table(a.b.kv_indptr, r, a.b.n_kv_blocks, a.b.max_blocks);
    const float rep = a.u.repetition ? a.u.repetition[r] : 1.f;
    const float pres = a.u.presence ? a.u.presence[r] : 0.f;
    const float freq = a.u.frequency ? a.u.frequency[r] : 0.f;
    const int prompt = a.u.prompt_len ? a.u.prompt_len[r] : 0;
    tkv::RowTable bias{0, 0, true};
    if (BIAS) bias = tkv::row_table(a.u.bias_indptr, r, a.u.n_bias, a.u.n_bias);
    const int first = a.search ? g - t.q0 : g / a.b.n_rows * a.per;
    if (!t.ok || first >= t.L) return;
    const int32_t early = BIAS && tid < bias.n ? a.u.bias_token[bias.first + tid] : -1;
    const int end = a.search ? first + 1 : min(t.L, first + a.per);
    const int c0 = tile * kTile, n = min(kTile, a.vocab - c0);
    const char* in = static_cast<const char*>(a.in) + (static_cast<int64_t>(t.q0 + first) * a.in_stride + c0) * (IN16 ? 2 : 4);
    char* out = static_cast<char*>(a.out) + (static_cast<int64_t>(t.q0 + first) * a.out_stride + c0) * (OUT16 ? 2 : 4);
    const int64_t in_step = a.in_stride * (IN16 ? 2 : 4), out_step = a.out_stride * (OUT16 ? 2 : 4);
    const bool ok = tab.ok && bias.ok && rep >= 0x1p-126f && rep <= 0x1p126f && fabsf(pres) < INFINITY && fabsf(freq) < INFINITY;
    const bool counts = ok && (rep != 1.f || pres != 0.f || freq != 0.f);
    const bool biased = BIAS && ok && bias.n > 0;

    // a thread a run of entries, kBatch of them at once; the first one's tokens are on their way before it is known where the run
    // begins in the path
    const int run = (tab.n + kThreads - 1) / kThreads;
    const int e0 = tab.first + min(tid * run, tab.n), e1 = tab.first + min(tid * run + run, tab.n);
    int id[kBatch], len[kBatch], keys = 0;
    const auto look = [&](int e) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) id[k] = e + k < e1 ? a.b.kv_blocks[e + k] : -1;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const bool there = static_cast<uint32_t>(id[k]) < static_cast<uint32_t>(a.num_blocks);
            len[k] = there ? a.b.block_len[id[k]] : 0;
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) len[k] = len[k] >= 1 && len[k] <= tkv::kBlock ? len[k] : 0;
    };
    i32x4_t tok[4];  // the next entry's tokens
    const auto fetch = [&](int block, int m) __attribute__((always_inline)) {
        if (m == 0) return;
        const i32x4_t* p = reinterpret_cast<const i32x4_t*>(a.tokens + static_cast<int64_t>(block) * tkv::kBlock);
#pragma unroll
        for (int q = 0; q < 4; ++q) tok[q] = p[q];
    };
    if (counts) {
        for (int e = e0 + (run - 1) / kBatch * kBatch; e >= e0; e -= kBatch) {  // the first ones last: they stay
            look(e);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) keys += len[k];
        }
        fetch(id[0], len[0]);
    }
    // a query token's logits, its grammar's words, and which of this thread's drafted tokens it sees
    f32x4_t x[kLoads];
    uint32_t words[kLoads], sees;
    bool fine, masked;
    const auto ask = [&](int i) __attribute__((always_inline)) {
        if (a.past_in) {
            asm volatile("");  // (as for the stores)
#pragma unroll
            for (int k = 0; k < kLoads; ++k) x[k] = load4<IN16, true>(in, (k * kThreads + tid) * 4, n);
            asm volatile("");
        } else {
#pragma unroll
            for (int k = 0; k < kLoads; ++k) x[k] = load4<IN16, false>(in, (k * kThreads + tid) * 4, n);
        }
        const int64_t q = t.q0 + i;
        // (asked for behind the logits, which it then waits for: ahead of them, 1,000 rows take 247 us for 230)
        const int grammar = a.u.grammar ? a.u.grammar[q] : -1;
        fine = ok && grammar < a.u.n_grammars;
        masked = fine && grammar >= 0;
        if (masked) {
            const uint32_t* allowed = a.u.allowed + static_cast<int64_t>(grammar) * a.u.allowed_words;
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                const int c = (k * kThreads + tid) * 4;
                if (c < n) words[k] = allowed[(c0 + c) >> 5];
            }
        }
        sees = 0;
        if (counts) {
            const uint64_t* mask = a.b.mask + q * a.b.mask_words;
            if (t.L == 1)
                sees = static_cast<uint32_t>(mask[0] & 1);
            else
                for (int j = tid, b = 0; j < t.L; j += kThreads, ++b) sees |= static_cast<uint32_t>(mask[j >> 6] >> (j & 63) & 1) << b;
        }
    };
    ask(first);
    if (counts) {
        count.clear(tid, kThreads);
        for (int j = tid; j < t.L; j += kThreads) drafted[j] = -1;
    }
    if (biased) given.clear(tid, kThreads);
    if (biased && !counts) __syncthreads();
    if (counts) {
        int N;
        int number = tkv::group_before<kWaves>(keys, N, part);  // (its barrier is the one after the clearing)
        const int context = t.L == 1 && sees ? N : N - t.L;  // (a single token counts or does not)
        // the tokens of an entry whose bits are set, by what is done with each of them
        const auto every = [&](const i32x4_t (&x)[4], uint32_t others, auto what) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const uint32_t other = static_cast<uint32_t>(static_cast<int32_t>(others << (31 - q)) >> 31);
                const uint32_t at = (static_cast<uint32_t>(x[q >> 2][q & 3]) - static_cast<uint32_t>(c0)) | other;
                if (at < static_cast<uint32_t>(n)) what(at, q);
            }
        };
        for (int e = 0; e < run; e += kBatch) {
            if (e > 0) {
                look(e0 + e);
                fetch(id[0], len[0]);
            }
            // (not unrolled: the instructions of one entry are 3 KB, and first reads of them are waited for)
#pragma unroll 1
            for (int k = 0; k < kBatch && e + k < run; ++k) {
                const int m = k == 0 ? len[0] : k == 1 ? len[1] : k == 2 ? len[2] : len[3];
                i32x4_t now[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) now[q] = tok[q];
                if (k + 1 < kBatch) fetch(k == 0 ? id[1] : k == 1 ? id[2] : id[3], k == 0 ? len[1] : k == 1 ? len[2] : len[3]);
                const int sure = min(max(context - number, 0), m);
                // (prompt is any number: a difference that cuts off where it would leave 32 bits)
                const int old = min(max(__builtin_elementwise_sub_sat(prompt, number), 0), sure);
                if (old < sure) every(now, ~((1u << sure) - (1u << old)), [&](uint32_t at, int) { count.more(at); });
                if (old > 0) every(now, ~((1u << old) - 1), [&](uint32_t at, int) { count.set(at); });
                if (sure < m && t.L > 1)
                    every(now, ~((1u << m) - (1u << sure)), [&](uint32_t at, int q) {
                        drafted[number + q - context] = static_cast<int32_t>(at) | (number + q >= prompt ? kPast : 0);
                    });
                number += m;
            }
        }
    }
    if (biased) {
        for (int e = tid; e < bias.n; e += kThreads) {
            const uint32_t at = static_cast<uint32_t>(e == tid ? early : a.u.bias_token[bias.first + e]) - static_cast<uint32_t>(c0);
            if (at < static_cast<uint32_t>(n)) given.raise(at, static_cast<uint32_t>(e) + 1);
        }
    }
    if (counts || biased) __syncthreads();

    const float inv = 1.f / rep;
    for (int i = first;;) {
        const bool tree = counts && t.L > 1;
        uint32_t put = 0;  // which of this thread's drafted tokens were the first to be seen in the prompt
        if (tree) {
            for (int j = tid, b = 0; j < t.L; j += kThreads, ++b) {
                const int32_t d = drafted[j];
                if (d < 0 || !(sees >> b & 1)) continue;
                if (d & kPast)
                    count.more(d & ~kPast);
                else if (count.mark(d))
                    put |= 1u << b;
            }
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int c = (k * kThreads + tid) * 4;
            if (c >= n) continue;
            f32x4_t y = x[k];
            if (counts) {
                uint32_t s[4];
                count.four(c, s);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (s[e] != 0) y[e] = y[e] > 0.f ? y[e] * inv : y[e] * rep;
                    const uint32_t times = s[e] & Cell::kTimes;
                    if (times != 0) y[e] = y[e] - freq * static_cast<float>(times) - pres;
                }
            }
            if (biased) {
                uint32_t w[4];
                given.four(c, w);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (w[e] != 0) y[e] += a.u.bias_value[bias.first + static_cast<int>(w[e]) - 1];
            }
            if (masked) {
                const uint32_t bits = words[k] >> ((c0 + c) & 31);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!(bits >> e & 1)) y[e] = -INFINITY;
            }
            if (!fine) y = f32x4_t{NAN, NAN, NAN, NAN};
            store4<OUT16>(out, c, n, y, a.past_out);
        }
        if (++i == end) break;
        in += in_step, out += out_step;
        const uint32_t seen = sees;
        ask(i);
        if (tree) {
            __syncthreads();
            for (int j = tid, b = 0; j < t.L; j += kThreads, ++b) {
                const int32_t d = drafted[j];
                if (d < 0 || !(seen >> b & 1)) continue;
                if (d & kPast)
                    count.less(d & ~kPast);
                else if (put >> b & 1)
                    count.unmark(d);
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
    const int64_t logits = static_cast<int64_t>(f.vocab) * f.b.n_qtok, out_bytes = logits * (f.out16 ? 2 : 4);
    a.past_out = out_bytes >= kPastOut;
    a.past_in = out_bytes + logits * (f.in16 ? 2 : 4) >= kPastIn;
    // The query tokens of a tree that share a workgroup's counts: few enough that 4,096 workgroups are left.  (64 trees of 16 to 32
    // tokens, 152,064, bf16 to fp32: one 397 us, two 378, four 355, eight 344; 319 by this rule, 327 with 2,048 left.)  With one, a
    // workgroup finds its token's row, so that none is without work in rows shorter than max_q.
    const int64_t tiles = static_cast<int64_t>(a.n_tiles) * f.b.n_qtok;
    a.per = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(8, f.b.max_q), tiles / 4096)));
    a.groups = (f.b.max_q + a.per - 1) / a.per;
    // Groups go by max_q: where it is far above the rows' tokens (a captured call's, say) most have no work, and a group a token is
    // faster.  (Those 64 trees under a max_q of 256, 1.3 groups a token: 334 us, 382 by tokens; 1,024, 5.2: 488 and 374.  300 rows of
    // up to 8 tokens under 64, 2.4: 316 and 345; 64 rows of up to 12 under 1,024, 62: 825 and 137.)
    if (static_cast<int64_t>(a.groups) * f.b.n_rows > 4 * static_cast<int64_t>(f.b.n_qtok)) a.per = 1;
    a.search = f.b.max_q > 1 && a.per == 1;
    int64_t all = a.search ? f.b.n_qtok : static_cast<int64_t>(a.groups) * f.b.n_rows;
    const int64_t most = (all + 7) / 8 * 8 * a.n_tiles;
    if (most > static_cast<int64_t>(UINT32_MAX) / 512)
        return set_error(TKV_EINVAL, "tkv_adjust_logits: %lld workgroups are too many", static_cast<long long>(most));
    a.units = static_cast<int32_t>(all);
    a.spread = all >= 64;  // (fewer units would leave XCDs without work at the end)
    if (a.spread) all = (all + 7) / 8 * 8;
    // Numbers of 32 bits where a path or a list of biases can pass 16, and where two workgroups a CU are enough: they take fewer
    // instructions, but 64 KB of LDS for the two instead of 32.  (Bf16 rows of 151,936 with paths of 200 to 4,000 tokens, in 32 and
    // 16 bits: 152 workgroups 9.2 and 9.3 us, 494 11.9 and 12.2, 570 16.1 and 14.3; 304 with paths of 8,000 to 30,000 14.6 and 16.0.)
    // 512 threads up to three workgroups a CU, 256 beyond: 646 13.9 and 14.6 us, 760 14.3 and 15.1, 1,026 19.0 and 18.2.
    const int64_t workgroups = all * a.n_tiles;
    const bool bias = f.u.n_bias > 0, wide = workgroups <= 512 || f.b.max_blocks > 0x7fff / kBlock || f.u.n_bias >= 0xffff;
    const bool many = workgroups >= 768;
    const auto run = [&](auto kernel, int threads) {
        kernel<<<dim3(static_cast<unsigned>(workgroups)), dim3(threads), 0, st>>>(a);
    };
    const auto typed = [&](auto has_bias, auto is_wide, auto n_threads) {
        constexpr bool B = decltype(has_bias)::value, W = decltype(is_wide)::value;
        constexpr int T = decltype(n_threads)::value;
        if (f.in16)
            f.out16 ? run(adjust<true, true, B, W, T>, T) : run(adjust<true, false, B, W, T>, T);
        else
            f.out16 ? run(adjust<false, true, B, W, T>, T) : run(adjust<false, false, B, W, T>, T);
    };
    const auto sized = [&](auto has_bias) {
        if (wide)
            typed(has_bias, std::true_type{}, std::integral_constant<int, 512>{});
        else if (many)
            typed(has_bias, std::false_type{}, std::integral_constant<int, 256>{});
        else
            typed(has_bias, std::false_type{}, std::integral_constant<int, 512>{});
    };
    bias ? sized(std::true_type{}) : sized(std::false_type{});
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TKV_OK : set_error(TKV_EHIP, "tkv_adjust_logits launch: %s", hipGetErrorString(e));
}
