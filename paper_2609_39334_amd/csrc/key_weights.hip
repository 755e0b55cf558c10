// The attention weight that a batch's queries give each key (tkv_key_weights): for key x of a row and KV head g
//   w'[x] = decay w[x] [x is context] + sum over the tokens i that see x of coef_i sum over the heads h of g of
//           exp(q_ih . k_x / sqrt(d) - lse_ih),
// with lse from the attention call before.  S = Q K^T runs on v_mfma_f32_32x32x16_bf16 with the queries as its rows, so that a
// lane holds one key's scores against 16 queries and their sum stays in the lane; K goes from the pool straight into the
// operand.  The coefficient goes into the exponent (lse - log c, infinite where nothing counts).  A key of a row and head
// belongs to one wave, in weigh_split to one workgroup, whose order of additions is fixed: no atomics.  The kernels' orders
// differ, and which one runs follows from the call's sizes: the same row may get other last bits in a call of other sizes.
//
// A call has to read each key once (2 d bytes a KV head) and two floats a key are read and written; it multiplies 2 d hq times and
// takes hq exponentials a key and token.  Few tokens are bound by memory, many by their exponentials and products.
//
// Three kernels.  weigh_few: rows of up to 32 queries a KV head (single tokens, small drafts) hold the queries in registers and
// stream K, the next 32 keys on their way.  weigh_many: 64 keys a wave stay in registers, and the queries pass in tiles of 32
// through LDS, double-buffered, shared by the four waves.  weigh_split: where there are few keys, the tiles are shared out among
// the waves.  Up to 32 queries the first is faster: 64 single tokens under 300 to 6,144 keys (12/2/128 heads) 24 us, 36 by the
// second; 1,000 tokens under 30 to 300 keys 29 and 45; 28/4 heads 27 and 36.
//
// Measured (times of calls one after the other): those 64 tokens 23 us, 102 MB, 4.5 TB/s.  32 tokens under one path of 30,000
// keys, 28/4/128: 17 us; 472 workgroups are less than two a CU, so it is a workgroup's own time: about 6 us until its first
// product (table, lengths, keys and first queries, a chain) and seven tiles of 1 us, 1.5 where there are masks.  8 rows of 64 to
// 256 tokens under 2,000 to 12,000 keys, 32/8/128 (67.8 GFLOP): 100 to 104 us, 650 to 675 TFLOP/s; MFMAs were busy 29% and the vector units 50%
// of the counted cycles (a product of 32 x 64 scores is 512 cycles of a SIMD's MFMAs, its exponentials 512 of a quarter-rate unit and about as
// many of others). Tried there, against 119 to 123 at the time: eight waves of 32 keys (123), two groups of keys one after the
// other in a workgroup (141), three waves a SIMD (127 to 133, registers spill in the steps), chunks slowest in the grid (130 to
// 141), products alone (103).  Masks tested score by score in a step of its own took 1.8 us a tile and these two calls 19.4 and
// 111 us; a lane's key has one word a tile instead, a bit a row, looked up for eight tiles at once and laid over the exponentials.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "internal.h"
#include "rows.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256, kWaves = 4;
// Most entries a workgroup of weigh_few, and workgroups aimed at: three a CU, what their registers allow.  (64 tokens under 300
// to 6,144 keys: 600 workgroups 26.2 us, 768 24.2, 1,024 27.0, 1,536 28.7.  Arrays ten times as long as the tables in them, as a
// captured call may have: 36 us, 178 without the limit.)
constexpr int kFewChunk = 64, kFewGroups = 768;
constexpr int kManyChunk = 16;    // entries a workgroup of weigh_many
constexpr int kSplitChunk = 4;    // entries a workgroup of weigh_split
constexpr int kSplitGroups = 512; // most workgroups of weigh_split: two a CU
constexpr int kWords = 9, kSplitWords = 3;  // words of 32 bits that 256 and 64 consecutive bits can touch
constexpr int kAhead = 8;         // tiles whose masks are looked up together
constexpr int kTokens = 8;        // tokens whose masks are read together
constexpr float kLog2e = 1.4426950408889634f;

struct Args {
    tkv_draft_batch b;
    int32_t num_blocks, hq, hkv, G, chunk, n_chunks;  // entries a chunk, chunks of the longest table
    bool search;                                      // units are counted over the rows
    uint32_t inv_g;                                   // 2^31 / G, rounded up
    float sl2, decay;                                 // log2(e) / sqrt(d)
    const uint16_t *q, *k;
    const float *lse, *coef, *before;
    float* out;
    int64_t keys;  // of a row and head in before and out
};

// What a workgroup works on: a chunk of a row's table, and a KV head.
struct Unit {
    int r, g, e0;
    tkv::RowTokens t;
    tkv::RowTable tab;
    bool ok;
};
__device__ __forceinline__ Unit unit_of(const Args& a) {
    Unit u;
    u.r = -1;
    int x = blockIdx.x;
    if (!a.search) {
        u.e0 = (a.n_chunks - 1 - x % a.n_chunks) * a.chunk;  // (a row's last keys, with masks, first)
        x /= a.n_chunks;
        u.g = x % a.hkv, u.r = x / a.hkv;
    } else {
        // the rows' chunks are counted up to this one, four rows a lane, by every wave for itself
        const int lane = threadIdx.x & 63;
        int64_t before = 0;
        for (int r0 = 0; r0 < a.b.n_rows && u.r < 0; r0 += 256) {
            int n[4], sum = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = r0 + 4 * lane + k;
                n[k] = 0;
                if (r < a.b.n_rows && tkv::row_tokens(a.b, r).ok)
                    n[k] = (tkv::row_table(a.b.kv_indptr, r, a.b.n_kv_blocks, a.b.max_blocks).n + a.chunk - 1) / a.chunk * a.hkv;
                sum += n[k];
            }
            int total;
            int64_t at = before + tkv::wave_before(sum, total);
            int mine = -1, left = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (x >= at && x < at + n[k]) mine = r0 + 4 * lane + k, left = static_cast<int>(x - at);
                at += n[k];
            }
            const uint64_t who = __builtin_amdgcn_ballot_w64(mine >= 0);
            if (who != 0) {
                const int l = __builtin_ctzll(who);
                u.r = __shfl(mine, l);
                left = __shfl(left, l);
                u.g = left % a.hkv, u.e0 = left / a.hkv * a.chunk;
            }
            before += total;
        }
        u.r = __builtin_amdgcn_readfirstlane(u.r);
    }
    u.ok = u.r >= 0;
    if (!u.ok) return u;
    u.t = tkv::row_tokens(a.b, u.r);
    u.tab = tkv::row_table(a.b.kv_indptr, u.r, a.b.n_kv_blocks, a.b.max_blocks);
    u.ok = u.t.ok && u.tab.ok && u.e0 < u.tab.n;
    return u;
}

// A thread's part of a chunk's table, in two steps so that other loads can go between: the block and length of entry `tid` of
// the chunk's n (at most as many as threads), and the length of entry `tid` behind it.
struct Look {
    int id, behind, len, more;
};
__device__ __forceinline__ void look_ids(const Args& a, const Unit& u, int n, Look& k) {
    const int tid = threadIdx.x, mine = u.e0 + tid, later = u.e0 + n + tid;
    k.id = tid < n && mine < u.tab.n ? a.b.kv_blocks[u.tab.first + mine] : -1;
    k.behind = tid < u.t.L && later < u.tab.n ? a.b.kv_blocks[u.tab.first + later] : -1;
}
__device__ __forceinline__ void look_lens(const Args& a, Look& k) {
    k.len = 0, k.more = 0;
    if (static_cast<uint32_t>(k.id) < static_cast<uint32_t>(a.num_blocks)) k.len = a.b.block_len[k.id];
    if (static_cast<uint32_t>(k.behind) < static_cast<uint32_t>(a.num_blocks)) k.more = a.b.block_len[k.behind];
}
// The chunk's blocks: {id, 32 (first key's number among the drafted ones, at least -64) + length}.  Ends in a barrier.
__device__ __forceinline__ void list_blocks(const Args& a, const Unit& u, int n, const Look& k, int2* list, int* part) {
    const int tid = threadIdx.x, step = min(kThreads, u.t.L);
    const int len = k.len >= 1 && k.len <= tkv::kBlock ? k.len : 0, more = k.more >= 1 && k.more <= tkv::kBlock ? k.more : 0;
    int total;
    const int before = tkv::group_before<kWaves>(more << 16 | len, total, part) & 0xffff;
    // keys behind the chunk, exact below the row's tokens
    int after = total >> 16;
    for (int next = u.e0 + n + step; after < u.t.L && next < u.tab.n; next += step) {
        int other, sum = 0;
        __syncthreads();
        if (tid < step && next + tid < u.tab.n)
            sum = tkv::entry_len(a.b.kv_blocks, a.b.block_len, a.num_blocks, u.tab.first + next + tid, other);
        tkv::group_before<kWaves>(sum, sum, part);
        after += sum;
    }
    if (tid < n) list[tid] = int2{k.id, 32 * max(u.t.L - (after + (total & 0xffff) - before), -64) + len};
    __syncthreads();
}

// Query row qr of a (row, KV head) is head qr % G of token qr / G (rows below 2^16, G at most 64).
__device__ __forceinline__ int token_of(const Args& a, int qr) {
    return static_cast<int>(__umulhi(static_cast<uint32_t>(2 * qr), a.inv_g));
}

// What is subtracted from a query row's score, in units of log2: infinite for a row that gives nothing (the logarithm of a
// coefficient below 2^-126 is -infinity).
__device__ __forceinline__ float offset_of(float z, float c) {
    float x = z * kLog2e - __builtin_amdgcn_logf(c);
    asm volatile("" : "+v"(x));  // (computed in any case: a branch would end the block that the compiler schedules as one)
    return fabsf(z) < INFINITY && c > 0.f ? x : INFINITY;
}

// All bits as bit i of x.
__device__ __forceinline__ uint32_t every_bit(uint32_t x, int i) {
    return static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(x), i, 1));
}

// Which of a tile's rows see a key that its tokens' bit `bit` of bits[token * words + word] stands for.
__device__ __forceinline__ uint32_t rows_that_see(const Args& a, int tile, int rows, const uint32_t* bits, int words, int word,
                                                  int bit) {
    const int from = token_of(a, 32 * tile), to = token_of(a, min(32 * tile + 31, rows - 1));
    const uint64_t group = ~0ull >> (64 - a.G);  // a token's rows, from its first one at `at` of the tile
    int at = from * a.G - 32 * tile;
    const uint32_t* m = bits + from * words + word;
    uint32_t s = every_bit(*m, bit) & static_cast<uint32_t>(group >> -at);
    m += words;
    for (int i = from + 1; i <= to; i += kTokens, m += kTokens * words) {
#pragma unroll
        for (int k = 0; k < kTokens; ++k) {  // (tokens behind the tile's last have no rows here, or masks of zeros)
            at += a.G;
            s |= every_bit(m[k * words], bit) & static_cast<uint32_t>(group << min(at, 32));
        }
    }
    return s;
}

// The first drafted key of a chunk of n entries (at most 64), -1: it has none.  Lane l looks at entry l.
__device__ __forceinline__ int first_drafted_of(const int2* list, int n) {
    const int lane = threadIdx.x & 63, d = list[min(lane, n - 1)].y, first = d >> 5, len = d & 31;
    const uint64_t has = __builtin_amdgcn_ballot_w64(lane < n && len > 0 && first + len > 0);
    return has != 0 ? max(__builtin_amdgcn_readlane(first, __builtin_ctzll(has)), 0) : -1;
}

// The tokens' masks from word w0 on, `words` words each, to bits, and kTokens masks of zeros behind them: a row's last tile may end
// inside, and its rows past the last token must not be seen to see (their products are 0 K, which is not 0 under any K).
template <int W>
__device__ __forceinline__ void stage_masks(const Args& a, const Unit& u, int w0, uint32_t* bits) {
    const int64_t words = 2 * static_cast<int64_t>(a.b.mask_words);
    const uint32_t* masks = reinterpret_cast<const uint32_t*>(a.b.mask) + u.t.q0 * words;
    const int given = u.t.L * W, n = given + kTokens * W;
    for (int m0 = threadIdx.x; m0 < n; m0 += 4 * kThreads) {
        uint32_t x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int m = m0 + k * kThreads, w = w0 + m % W;
            x[k] = m < given && w < words ? masks[m / W * words + w] : 0;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (m0 + k * kThreads < n) bits[m0 + k * kThreads] = x[k];
    }
}

template <int D>
__global__ __launch_bounds__(kThreads, 3) void weigh_few(Args a) {
    constexpr int KS = D / 16;
    __shared__ int2 list[kFewChunk];
    __shared__ int part[kWaves];
    const Unit u = unit_of(a);
    if (!u.ok) return;
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, hi = lane >> 5;
    const int rows = u.t.L * a.G, nu = (rows + 7) / 8;
    Look look;
    look_ids(a, u, a.chunk, look);
    bf16x8_t qf[KS];
    {
        const int qr = min(col, rows - 1), i = token_of(a, qr);
        const uint16_t* row = a.q + (static_cast<int64_t>(u.t.q0 + i) * a.hq + u.g * a.G + (qr - i * a.G)) * D + 8 * hi;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const bf16x8_t*>(row + 16 * s);
    }
    look_lens(a, look);
    // x[4 v + e] of a product is query row 8 v + 4 hi + e
    float off[16];
    uint32_t mask;  // of row `col`: a row's tokens are at most 32
    {
        const int qr = min(col, rows - 1), i = token_of(a, qr);
        const int64_t token = u.t.q0 + i;
        const float z = a.lse[token * a.hq + u.g * a.G + (qr - i * a.G)], c = a.coef ? a.coef[token] : 1.f;
        mask = col < rows ? static_cast<uint32_t>(a.b.mask[token * a.b.mask_words]) : 0;
        const float mine = col < rows ? offset_of(z, c) : INFINITY;
        if (mine == INFINITY) {  // a row that gives nothing may hold anything
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[s] = bf16x8_t{};
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) off[e] = __shfl(mine, 8 * (e >> 2) + 4 * hi + (e & 3));
    }
    const int n = min(a.chunk, u.tab.n - u.e0), pairs = (n + 1) / 2;
    list_blocks(a, u, a.chunk, look, list, part);

    float* out = a.out + (static_cast<int64_t>(u.r) * a.hkv + u.g) * a.keys + 16 * static_cast<int64_t>(u.e0);
    const float* before = a.before ? a.before + (out - a.out) : nullptr;
    const auto fetch = [&](int p, bf16x8_t (&kf)[KS], int2& d, float& had) {
        d = p < pairs ? list[min(2 * p + (col >> 4), a.chunk - 1)] : int2{0, 32 * -64};
        if (2 * p + (col >> 4) >= n) d.y = 32 * -64;
        had = 0.f;
        if ((col & 15) < (d.y & 31)) {
            const uint16_t* row = a.k + (static_cast<int64_t>(d.x) * a.hkv + u.g) * (16 * D) + (col & 15) * D + 8 * hi;
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[s] = *reinterpret_cast<const bf16x8_t*>(row + 16 * s);
            if (before && hi == 0) had = before[32 * p + col];
        }
    };
    const auto weigh = [&](int p, const bf16x8_t (&kf)[KS], int2 d, float had) {
        const int slot = col & 15, j = (d.y >> 5) + slot;  // this lane's key among the drafted ones (negative: context)
        const bool there = slot < (d.y & 31);
        f32x16_t x{};
#pragma unroll
        for (int s = 0; s < KS; ++s) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[s], kf[s], x, 0, 0, 0);
        float sum = 0.f;
        if (__builtin_amdgcn_ballot_w64(there && j >= 0) == 0) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (v < nu) {
#pragma unroll
                    for (int e = 4 * v; e < 4 * v + 4; ++e) sum += __builtin_amdgcn_exp2f(fmaf(x[e], a.sl2, -off[e]));
                }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t row = __shfl(mask, 8 * (e >> 2) + 4 * hi + (e & 3));
                const float w = __builtin_amdgcn_exp2f(fmaf(x[e], a.sl2, -off[e]));
                sum += there && (j < 0 || (row >> (j & 31) & 1)) ? w : 0.f;
            }
        }
        sum += __shfl_xor(sum, 32);
        if (there && hi == 0) out[32 * p + col] = j < 0 ? fmaf(a.decay, had, sum) : sum;
    };
    bf16x8_t k0[KS], k1[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) k0[s] = bf16x8_t{}, k1[s] = bf16x8_t{};
    int2 d0, d1;
    float h0, h1;
    fetch(wid, k0, d0, h0);
    for (int p = wid; p < pairs; p += 2 * kWaves) {
        fetch(p + kWaves, k1, d1, h1);
        weigh(p, k0, d0, h0);
        fetch(p + 2 * kWaves, k0, d0, h0);
        if (p + kWaves < pairs) weigh(p + kWaves, k1, d1, h1);
    }
}

// (Three waves a SIMD for heads of 64: 32 rows of 40 to 100 tokens, eight heads of their own, 22 us, 25 with two; ten values are
// spilled ahead of the steps under masks and come back behind them.)
template <int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void weigh_many(Args a) {
    constexpr int KS = D / 16, CPR = D / 8, kPieces = 32 * CPR / kThreads;  // 16-byte pieces a row, pieces of a tile a thread
    __shared__ __attribute__((aligned(16))) uint16_t qs[2][32 * D];
    __shared__ __attribute__((aligned(16))) float offs[4][32];
    extern __shared__ uint32_t bits[];  // the tokens' masks from the chunk's first drafted key on, kWords each
    __shared__ uint32_t seen[kWaves][kAhead][64];  // tile t's at t % kAhead: which of its rows see each of a wave's keys
    __shared__ int2 list[kManyChunk];
    __shared__ int part[kWaves];
    const Unit u = unit_of(a);
    if (!u.ok) return;
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hi = lane >> 5;
    const int rows = u.t.L * a.G, n_tiles = (rows + 31) / 32;

    // a tile of 32 query rows, their 16-byte pieces XOR-swizzled by row so that the operand reads meet no bank conflict; two tiles
    // are on their way (tile t in set t % 2), and what follows from their loads is left until these are back
    u32x4_t qx[2][kPieces];
    float zx[2], cx[2];  // of row `col`
    const uint16_t* q0 = a.q + (static_cast<int64_t>(u.t.q0) * a.hq + u.g * a.G) * D + tid % CPR * 8;
    const float* lse = a.lse + static_cast<int64_t>(u.t.q0) * a.hq + u.g * a.G;
    const float* coef = a.coef ? a.coef + u.t.q0 : lse;  // (lse where there are none: its values are masked out)
    const uint32_t given = a.coef ? ~0u : 0u;
    const auto fetch_q = [&](int tile, int set) __attribute__((always_inline)) {
#pragma unroll
        for (int y = 0; y < kPieces; ++y) {
            const int qr = min(32 * tile + (y * kThreads + tid) / CPR, rows - 1), i = token_of(a, qr);
            qx[set][y] = *reinterpret_cast<const u32x4_t*>(q0 + (i * (a.hq - a.G) + qr) * D);  // (below 2^10 256 128 elements)
        }
        // (every wave reads the rows' lse and coefficients, so that a step has no branches)
        const int qr = min(32 * tile + col, rows - 1), i = token_of(a, qr);
        zx[set] = lse[i * (a.hq - a.G) + qr];
        cx[set] = coef[i];
    };
    // the table first, then its lengths, then the keys (rows past a block's length are read, and nothing made of them): loads
    // come back in order.  (K is read in four pieces of 32 bytes a line: past the caches each piece is fetched for itself, 40 us
    // for 25.)
    Look look;
    look_ids(a, u, kManyChunk, look);
    int own[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int e = u.e0 + 4 * wid + 2 * h + (col >> 4);
        own[h] = e < u.tab.n ? a.b.kv_blocks[u.tab.first + e] : -1;
    }
    fetch_q(0, 0);
    look_lens(a, look);
    bf16x8_t kf[2][KS];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[h][s] = bf16x8_t{};
        if (static_cast<uint32_t>(own[h]) < static_cast<uint32_t>(a.num_blocks)) {
            const uint16_t* row = a.k + (static_cast<int64_t>(own[h]) * a.hkv + u.g) * (16 * D) + (col & 15) * D + 8 * hi;
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[h][s] = *reinterpret_cast<const bf16x8_t*>(row + 16 * s);
        }
    }
    list_blocks(a, u, kManyChunk, look, list, part);

    // what is read and written is key 64 wid + lane of the chunk
    const int entry = 4 * wid + (lane >> 4), slot = lane & 15;
    const int64_t at = (static_cast<int64_t>(u.r) * a.hkv + u.g) * a.keys + 16 * static_cast<int64_t>(u.e0 + entry) + slot;
    const int number = (list[entry].y >> 5) + slot;
    const float had = slot < (list[entry].y & 31) && number < 0 && a.before ? a.before[at] : 0.f;
    const int first_drafted = first_drafted_of(list, kManyChunk);
    const auto put = [&](int tile, int set) __attribute__((always_inline)) {
        const float c = __uint_as_float((__float_as_uint(cx[set]) & given) | (__float_as_uint(1.f) & ~given));
        float off = offset_of(zx[set], c);
        off = 32 * tile + col < rows ? off : INFINITY;
        offs[tile & 3][col] = off;
        // a row that gives nothing may hold anything: zeros in its place
        const uint32_t none = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(off == INFINITY));
#pragma unroll
        for (int y = 0; y < kPieces; ++y) {
            const int x = y * kThreads + tid, row = x / CPR;
            const int swz = D == 128 ? row & 15 : (row >> 1) & 7;
            const uint32_t keep = (none >> row & 1) - 1;
            *reinterpret_cast<u32x4_t*>(qs[set] + row * D + ((x % CPR) ^ swz) * 8) = qx[set][y] & keep;
        }
    };
    const int swz = D == 128 ? col & 15 : (col >> 1) & 7;
    float sum[2] = {0.f, 0.f};
    // x[4 v + e] of a product is query row 8 v + 4 hi + e of the tile
    const auto multiply = [&](int tile, f32x16_t (&x)[2]) __attribute__((always_inline)) {
        const uint16_t* row = qs[tile & 1] + col * D;
        x[0] = f32x16_t{}, x[1] = f32x16_t{};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const bf16x8_t qf = *reinterpret_cast<const bf16x8_t*>(row + ((2 * s + hi) ^ swz) * 8);
#pragma unroll
            for (int h = 0; h < 2; ++h) x[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[h][s], x[h], 0, 0, 0);
        }
    };
    const auto add = [&](int tile, const f32x16_t (&x)[2], const uint32_t (&sees)[2], auto masked) __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const f32x4_t o = *reinterpret_cast<const f32x4_t*>(offs[tile & 3] + 8 * v + 4 * hi);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(fmaf(x[h][4 * v + e], a.sl2, -o[e]));
                    if (masked) p[e] = __uint_as_float(__float_as_uint(p[e]) & every_bit(sees[h], 8 * v + e));
                }
                sum[h] += (p[0] + p[1]) + (p[2] + p[3]);
            }
        }
    };
    // this lane's word of `seen` for tiles t to t + kAhead - 1, of key 64 wid + lane of the chunk
    int word = 0, bit = 0;
    uint32_t context = 0;
    const auto look_seen = [&](int t) {
        for (int tile = t; tile < min(t + kAhead, n_tiles); ++tile) {
            seen[wid][tile % kAhead][lane] = context | rows_that_see(a, tile, rows, bits, kWords, word, bit);
        }
    };
    // a tile's products beside the exponentials of the one before
    const auto walk = [&](auto masked) __attribute__((always_inline)) {
        f32x16_t x[2][2];
        uint32_t sees[2][2];
        const auto begin = [&](int t, int set) __attribute__((always_inline)) {
            if (masked) {
#pragma unroll
                for (int h = 0; h < 2; ++h) sees[set][h] = seen[wid][t % kAhead][32 * h + col] >> (4 * hi);
            }
            multiply(t, x[set]);
        };
        const auto step = [&](int t, int set) __attribute__((always_inline)) {  // set: t % 2
            fetch_q(t + 2, set);  // (tiles past the last read its last row again, and give nothing)
            if (masked && set == 0 && t % kAhead == 0) look_seen(t);
            __syncthreads();
            __builtin_amdgcn_sched_barrier(0);
            begin(t, set);
            add(t - 1, x[set ^ 1], sees[set ^ 1], masked);
            put(t + 1, set ^ 1);
        };
        put(0, 0);
        fetch_q(1, 1);
        fetch_q(2, 0);
        __syncthreads();
        if (masked) look_seen(0);
        begin(0, 0);
        put(1, 1);
        int t = 1;
        for (; t + 1 < n_tiles; t += 2) {
            step(t, 1);
            step(t + 1, 0);
        }
        if (t < n_tiles) {
            step(t, 1);
            add(t, x[1], sees[1], masked);
        } else {
            add(t - 1, x[0], sees[0], masked);
        }
    };
    if (first_drafted < 0) {
        walk(std::false_type{});
    } else {
        const int w0 = first_drafted >> 5;
        stage_masks<kWords>(a, u, w0, bits);
        context = number < 0 ? ~0u : 0;
        if (number >= 0 && slot < (list[entry].y & 31)) word = (number >> 5) - w0, bit = number & 31;
        walk(std::true_type{});
    }
    const float w0 = sum[0] + __shfl_xor(sum[0], 32), w1 = sum[1] + __shfl_xor(sum[1], 32);
    if (slot < (list[entry].y & 31)) a.out[at] = fmaf(a.decay, had, hi == 0 ? w0 : w1);
}

// weigh_many for few keys: 64 of them a workgroup, which all its waves hold, and a wave takes every fourth tile of queries, straight
// into the operand.  The waves' sums meet in LDS at the end, in their order.
template <int D>
__global__ __launch_bounds__(kThreads, 2) void weigh_split(Args a) {
    constexpr int KS = D / 16;
    extern __shared__ uint32_t bits[];  // the tokens' masks from the chunk's first drafted key on, kSplitWords each
    __shared__ __attribute__((aligned(16))) float offs[kWaves][32];
    __shared__ float sums[kWaves][64];
    __shared__ int2 list[kSplitChunk];
    __shared__ int part[kWaves];
    const Unit u = unit_of(a);
    if (!u.ok) return;
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hi = lane >> 5;
    const int rows = u.t.L * a.G, n_tiles = (rows + 31) / 32;
    const uint16_t* q0 = a.q + (static_cast<int64_t>(u.t.q0) * a.hq + u.g * a.G) * D + 8 * hi;
    const float* lse = a.lse + static_cast<int64_t>(u.t.q0) * a.hq + u.g * a.G;
    bf16x8_t qf[2][KS];
    float z[2], c[2];  // of row `col`
    const auto fetch_q = [&](int tile, int set) __attribute__((always_inline)) {
        const int qr = min(32 * tile + col, rows - 1), i = token_of(a, qr), head = i * (a.hq - a.G) + qr;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[set][s] = *reinterpret_cast<const bf16x8_t*>(q0 + head * D + 16 * s);  // (below 2^10 256 128)
        z[set] = lse[head];
        c[set] = a.coef ? a.coef[u.t.q0 + i] : 1.f;
    };
    Look look;
    look_ids(a, u, kSplitChunk, look);
    int own[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int e = u.e0 + 2 * h + (col >> 4);
        own[h] = e < u.tab.n ? a.b.kv_blocks[u.tab.first + e] : -1;
    }
    fetch_q(wid, 0);
    look_lens(a, look);
    bf16x8_t kf[2][KS];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[h][s] = bf16x8_t{};
        if (static_cast<uint32_t>(own[h]) < static_cast<uint32_t>(a.num_blocks)) {
            const uint16_t* row = a.k + (static_cast<int64_t>(own[h]) * a.hkv + u.g) * (16 * D) + (col & 15) * D + 8 * hi;
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[h][s] = *reinterpret_cast<const bf16x8_t*>(row + 16 * s);
        }
    }
    list_blocks(a, u, kSplitChunk, look, list, part);

    // what is read and written, and whose masks a lane looks up, is key `lane` of the chunk
    const int entry = lane >> 4, slot = lane & 15, number = (list[entry].y >> 5) + slot;
    const bool there = slot < (list[entry].y & 31);
    const int64_t at = (static_cast<int64_t>(u.r) * a.hkv + u.g) * a.keys + 16 * static_cast<int64_t>(u.e0 + entry) + slot;
    const float had = wid == 0 && there && number < 0 && a.before ? a.before[at] : 0.f;
    const int first_drafted = first_drafted_of(list, kSplitChunk);
    const bool masked = first_drafted >= 0;
    const uint32_t context = number < 0 ? ~0u : 0;
    int word = 0, bit = 0;
    if (masked) {
        const int w0 = first_drafted >> 5;
        stage_masks<kSplitWords>(a, u, w0, bits);
        if (number >= 0 && there) word = (number >> 5) - w0, bit = number & 31;
        __syncthreads();
    }
    float sum[2] = {0.f, 0.f};
    const auto step = [&](int t, int set) __attribute__((always_inline)) {
        fetch_q(t + kWaves, set ^ 1);  // (tiles past the last read its last row again)
        float off = offset_of(z[set], c[set]);
        off = 32 * t + col < rows ? off : INFINITY;
        if (off == INFINITY) {  // a row that gives nothing may hold anything
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[set][s] = bf16x8_t{};
        }
        offs[wid][col] = off;
        f32x16_t x[2] = {f32x16_t{}, f32x16_t{}};
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) x[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[set][s], kf[h][s], x[h], 0, 0, 0);
        uint32_t sees[2] = {~0u, ~0u};
        if (masked) {
            const uint32_t s = context | rows_that_see(a, t, rows, bits, kSplitWords, word, bit);
#pragma unroll
            for (int h = 0; h < 2; ++h) sees[h] = __shfl(s, 32 * h + col) >> (4 * hi);
        }
        // x[h][4 v + e] is query row 8 v + 4 hi + e of the tile
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const f32x4_t o = *reinterpret_cast<const f32x4_t*>(offs[wid] + 8 * v + 4 * hi);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(fmaf(x[h][4 * v + e], a.sl2, -o[e]));
                    p[e] = __uint_as_float(__float_as_uint(p[e]) & every_bit(sees[h], 8 * v + e));
                }
                sum[h] += (p[0] + p[1]) + (p[2] + p[3]);
            }
        }
    };
    for (int t = wid; t < n_tiles; t += 2 * kWaves) {
        step(t, 0);
        if (t + kWaves < n_tiles) step(t + kWaves, 1);
    }
    const float w0 = sum[0] + __shfl_xor(sum[0], 32), w1 = sum[1] + __shfl_xor(sum[1], 32);
    sums[wid][lane] = hi == 0 ? w0 : w1;
    __syncthreads();
    if (wid == 0 && there) a.out[at] = fmaf(a.decay, had, (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]));
}

}  // namespace

int tkv::launch_key_weights(const tkv_shape& s, const tkv_draft_batch& b, const void* q, const void* k, const float* lse,
                            const float* coef, float decay, const float* before, float* out, int64_t keys, void* stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    Args a{};
    a.b = b;
    a.num_blocks = s.num_blocks, a.hq = s.hq, a.hkv = s.hkv, a.G = s.hq / s.hkv;
    a.inv_g = ((1u << 31) + a.G - 1) / a.G;
    a.sl2 = kLog2e / sqrtf(static_cast<float>(s.d));
    a.decay = decay;
    a.q = static_cast<const uint16_t*>(q), a.k = static_cast<const uint16_t*>(k);
    a.lse = lse, a.coef = coef, a.before = decay != 0.f ? before : nullptr, a.out = out, a.keys = keys;
    const bool few = static_cast<int64_t>(b.max_q) * a.G <= 32;
    // weigh_split where its workgroups run all at once, two a CU, and a wave has a tile at least.  (32/4/128 heads, many and split: one
    // row of 3,550 keys and 32, 64, 128 tokens 13.9 and 9.1, 22.4 and 12.6, 40.2 and 17.9 us; two such rows, 458 workgroups, 15.1 and
    // 13.4, 23.7 and 18.7, 41.4 and 26.6; three rows 15.4 and 23.0, 24.2 and 30.4, 42.8 and 46.2.  Two rows of 16 tokens, four tiles,
    // 10.5 and 11.4; two tiles 7.1 and 9.1.  Nine rows of 200 tokens under 1,200 keys, 14/2/64: 55 and 24.)
    const bool split = !few && (static_cast<int64_t>(b.max_q) * a.G + 31) / 32 >= kWaves &&
                       (b.n_kv_blocks / kSplitChunk + static_cast<int64_t>(b.n_rows)) * s.hkv <= kSplitGroups;
    a.chunk = split ? kSplitChunk : kManyChunk;
    if (few) {
        const int64_t even = static_cast<int64_t>(b.n_kv_blocks) * s.hkv / kFewGroups;
        a.chunk = static_cast<int32_t>(std::max<int64_t>(8, std::min<int64_t>(kFewChunk, (even + 7) / 8 * 8)));
    }
    // Workgroup b runs on XCD b % 8: an odd number of chunks, or the rows' first chunks, which all rows have, would share one.
    a.n_chunks = (b.max_blocks + a.chunk - 1) / a.chunk | 1;
    // A workgroup finds its row by division where that leaves few without work, or counts the rows' chunks up to its own: one row of
    // 30,000 keys beside 300 of 30 to 300 takes 23 us counted and 75 divided, 1,000 rows of like lengths 52 and 29.
    const int64_t heads = static_cast<int64_t>(b.n_rows) * s.hkv, most = static_cast<int64_t>(UINT32_MAX) / kThreads;
    const int64_t direct = a.n_chunks * std::min(heads, most + 1);  // (2^25 2^24 at most)
    const int64_t counted = (b.n_kv_blocks / a.chunk + static_cast<int64_t>(b.n_rows)) * s.hkv;
    a.search = direct > 4 * counted;
    const int64_t grid = a.search ? counted : direct;
    if (grid > most || heads > most)
        return set_error(TKV_EINVAL, "tkv_key_weights: %lld workgroups are too many", static_cast<long long>(grid));
    const size_t lds = few ? 0 : static_cast<size_t>(b.max_q + kTokens) * (split ? kSplitWords : kWords) * 4;  // (62 KB with all)
    const auto run = [&](auto kernel) { kernel<<<dim3(static_cast<unsigned>(grid)), dim3(kThreads), lds, st>>>(a); };
    if (s.d == 128)
        few ? run(weigh_few<128>) : split ? run(weigh_split<128>) : run(weigh_many<128>);
    else
        few ? run(weigh_few<64>) : split ? run(weigh_split<64>) : run(weigh_many<64>);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TKV_OK : set_error(TKV_EHIP, "tkv_key_weights launch: %s", hipGetErrorString(e));
}
