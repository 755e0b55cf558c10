// The attention weight that a batch's queries give each key (tkv_key_weights): for key x of a row and KV head g
//   w'[x] = decay w[x] [x is context] + sum over the tokens i that see x of coef_i sum over the heads h of g of
//           exp(q_ih . k_x / sqrt(d) - lse_ih),
// with lse from the attention call before.  S = Q K^T runs on v_mfma_f32_32x32x16_bf16 with the queries as its rows, so that a
// lane holds one key's scores against 16 queries and their sum stays in the lane; K goes from the pool straight into the
// operand.  The coefficient goes into the exponent (lse - log c, infinite where nothing counts).  A key of a row and head
// belongs to one wave, whose order of additions is fixed: no atomics.
//
// Two kernels.  weigh_few: rows of up to 32 queries a KV head (single tokens, small drafts) hold the queries in registers and
// stream K, the next 32 keys on their way.  weigh_many: 64 keys a wave stay in registers, and the queries pass in tiles of 32
// through LDS, double-buffered, shared by the four waves.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cstdint>

#include "internal.h"
#include "rows.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kFewChunk = 256;    // most entries a workgroup of weigh_few
constexpr int kManyChunk = 16;    // entries a workgroup of weigh_many
constexpr int kWords = 9;         // words of 32 bits that 256 consecutive bits can touch
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

// The chunk's blocks: {id, 32 (first key's number among the drafted ones, at least -64) + length}; n: entries of the chunk, at
// most as many as threads.  Ends in a barrier.
__device__ __forceinline__ void list_blocks(const Args& a, const Unit& u, int n, int2* list, int* part) {
    const int tid = threadIdx.x, step = min(kThreads, u.t.L);
    const int mine = u.e0 + tid, later = u.e0 + n + tid;
    int id = -1, behind = -1, len = 0, more = 0, total;
    if (tid < n && mine < u.tab.n) id = a.b.kv_blocks[u.tab.first + mine];
    if (tid < step && later < u.tab.n) behind = a.b.kv_blocks[u.tab.first + later];
    if (static_cast<uint32_t>(id) < static_cast<uint32_t>(a.num_blocks)) len = a.b.block_len[id];
    if (static_cast<uint32_t>(behind) < static_cast<uint32_t>(a.num_blocks)) more = a.b.block_len[behind];
    len = len >= 1 && len <= tkv::kBlock ? len : 0;
    more = more >= 1 && more <= tkv::kBlock ? more : 0;
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
    if (tid < n) list[tid] = int2{id, 32 * max(u.t.L - (after + (total & 0xffff) - before), -64) + len};
    __syncthreads();
}

// Query row qr of a (row, KV head) is head qr % G of token qr / G (rows below 2^16, G at most 64).
__device__ __forceinline__ int token_of(const Args& a, int qr) {
    return static_cast<int>(__umulhi(static_cast<uint32_t>(2 * qr), a.inv_g));
}

// What is subtracted from a query row's score, in units of log2: infinite for a row that gives nothing.
__device__ __forceinline__ float offset_of(const Args& a, int64_t token, int head) {
    const float z = a.lse[token * a.hq + head], c = a.coef ? a.coef[token] : 1.f;
    return fabsf(z) < INFINITY && c > 0.f ? z * kLog2e - (a.coef ? log2f(c) : 0.f) : INFINITY;
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
    bf16x8_t qf[KS];
    {
        const int qr = min(col, rows - 1), i = token_of(a, qr);
        const uint16_t* row = a.q + (static_cast<int64_t>(u.t.q0 + i) * a.hq + u.g * a.G + (qr - i * a.G)) * D + 8 * hi;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const bf16x8_t*>(row + 16 * s);
    }
    // x[4 v + e] of a product is query row 8 v + 4 hi + e
    float off[16];
    {
        const int i = token_of(a, min(col, rows - 1));
        const float mine = col < rows ? offset_of(a, u.t.q0 + i, u.g * a.G + (col - i * a.G)) : INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) off[e] = __shfl(mine, 8 * (e >> 2) + 4 * hi + (e & 3));
    }
    const int n = min(a.chunk, u.tab.n - u.e0), pairs = (n + 1) / 2;
    list_blocks(a, u, a.chunk, list, part);

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
            uint32_t sees = 0;  // the rows that see this lane's key
#pragma unroll 1
            for (int e = 0; e < 4 * nu; ++e) {
                const int row = 8 * (e >> 2) + 4 * hi + (e & 3);
                if (there && row < rows &&
                    (j < 0 || a.b.mask[static_cast<int64_t>(u.t.q0 + token_of(a, row)) * a.b.mask_words + (j >> 6)] >> (j & 63) & 1))
                    sees |= 1u << e;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float w = __builtin_amdgcn_exp2f(fmaf(x[e], a.sl2, -off[e]));
                sum += sees >> e & 1 ? w : 0.f;
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

template <int D>
__global__ __launch_bounds__(kThreads, 3) void weigh_many(Args a) {
    constexpr int KS = D / 16, CPR = D / 8, kPieces = 32 * CPR / kThreads;  // 16-byte pieces a row, pieces of a tile a thread
    __shared__ __attribute__((aligned(16))) uint16_t qs[2][32 * D];
    __shared__ __attribute__((aligned(16))) float offs[2][32];
    __shared__ uint32_t bits[2][32][kWords];  // the rows' masks from the chunk's first drafted key on
    __shared__ int2 list[kManyChunk];
    __shared__ int part[kWaves];
    const Unit u = unit_of(a);
    if (!u.ok) return;
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hi = lane >> 5;
    const int rows = u.t.L * a.G, n_tiles = (rows + 31) / 32;

    // a tile of 32 query rows, their 16-byte pieces XOR-swizzled by row so that the operand reads meet no bank conflict
    u32x4_t qx[kPieces];
    float ox = 0.f;
    uint32_t bx[2] = {0, 0};
    const auto fetch_q = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int y = 0; y < kPieces; ++y) {
            const int x = y * kThreads + tid, qr = min(32 * tile + x / CPR, rows - 1), i = token_of(a, qr);
            qx[y] = *reinterpret_cast<const u32x4_t*>(a.q + (static_cast<int64_t>(u.t.q0 + i) * a.hq + u.g * a.G + (qr - i * a.G)) * D + x % CPR * 8);
        }
        if (tid < 32) {
            const int qr = 32 * tile + tid, i = token_of(a, min(qr, rows - 1));
            ox = qr < rows ? offset_of(a, u.t.q0 + i, u.g * a.G + (qr - i * a.G)) : INFINITY;
        }
    };
    fetch_q(0);
    list_blocks(a, u, kManyChunk, list, part);

    bf16x8_t kf[2][KS];
    int j[2], place[2];
    bool there[2];
    int low = INT32_MAX, high = -1;  // the wave's drafted keys
    bool context = false;            // whether it has others
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int e = 4 * wid + 2 * h + (col >> 4), slot = col & 15;
        const int2 d = list[e];
        there[h] = slot < (d.y & 31);
        j[h] = (d.y >> 5) + slot;
        place[h] = 16 * e + slot;
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[h][s] = bf16x8_t{};
        if (there[h]) {
            const uint16_t* row = a.k + (static_cast<int64_t>(d.x) * a.hkv + u.g) * (16 * D) + slot * D + 8 * hi;
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[h][s] = *reinterpret_cast<const bf16x8_t*>(row + 16 * s);
        }
    }
    int lowest = INT32_MAX;  // the chunk's first drafted key
    for (int e = kManyChunk - 1; e >= 0; --e) {
        const int first = list[e].y >> 5, len = list[e].y & 31;
        if (len == 0) continue;
        if (first + len > 0) lowest = max(first, 0);
        if (e >> 2 != wid) continue;
        if (first < 0) context = true;
        if (first + len > 0) low = max(first, 0), high = max(high, first + len - 1);
    }
    lowest = __builtin_amdgcn_readfirstlane(lowest), low = __builtin_amdgcn_readfirstlane(low);
    high = __builtin_amdgcn_readfirstlane(high), context = __builtin_amdgcn_readfirstlane(context);
    const bool some = lowest < INT32_MAX, drafted = high >= 0;
    const int w0 = some ? lowest >> 5 : 0;
    const auto fetch_bits = [&](int tile) __attribute__((always_inline)) {
        if (!some) return;
        const uint32_t* masks = reinterpret_cast<const uint32_t*>(a.b.mask);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int x = y * kThreads + tid, qr = 32 * tile + x / kWords, w = w0 + x % kWords;
            bx[y] = x < 32 * kWords && w < 2 * a.b.mask_words && qr < rows
                        ? masks[static_cast<int64_t>(u.t.q0 + token_of(a, qr)) * (2 * a.b.mask_words) + w] : 0;
        }
    };
    const auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int y = 0; y < kPieces; ++y) {
            const int x = y * kThreads + tid, row = x / CPR;
            const int swz = D == 128 ? row & 15 : (row >> 1) & 7;
            *reinterpret_cast<u32x4_t*>(qs[buf] + row * D + ((x % CPR) ^ swz) * 8) = qx[y];
        }
        if (tid < 32) offs[buf][tid] = ox;
        if (some) {
            bits[buf][tid / kWords][tid % kWords] = bx[0];
            if (tid + kThreads < 32 * kWords) bits[buf][(tid + kThreads) / kWords][(tid + kThreads) % kWords] = bx[1];
        }
    };
    const int swz = D == 128 ? col & 15 : (col >> 1) & 7;
    float sum[2] = {0.f, 0.f};
    fetch_bits(0);
    put(0);
    for (int t = 0; t < n_tiles; ++t) {
        const int buf = t & 1;
        if (t + 1 < n_tiles) fetch_q(t + 1), fetch_bits(t + 1);
        __syncthreads();
        // whether the tile's rows (padding aside) see all of the wave's drafted keys, or none
        bool all = true, none = false;
        if (drafted) {
            bool every = true, any = false;
            for (int w = low >> 5; w <= high >> 5; ++w) {
                const uint32_t from = w == low >> 5 ? ~0u << (low & 31) : ~0u, to = w == high >> 5 ? ~0u >> (31 - (high & 31)) : ~0u;
                const uint32_t seen = bits[buf][col][w - w0] & from & to;
                every = every && seen == (from & to), any = any || seen != 0;
            }
            all = __builtin_amdgcn_ballot_w64(!every && 32 * t + col < rows) == 0;
            none = !context && __builtin_amdgcn_ballot_w64(any && 32 * t + col < rows) == 0;
        }
        if (!none) {
            f32x16_t x0{}, x1{};
            const uint16_t* row = qs[buf] + col * D;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bf16x8_t qf = *reinterpret_cast<const bf16x8_t*>(row + ((2 * s + hi) ^ swz) * 8);
                x0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[0][s], x0, 0, 0, 0);
                x1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[1][s], x1, 0, 0, 0);
            }
            // x[4 v + e] is query row 8 v + 4 hi + e of the tile
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const f32x4_t o = *reinterpret_cast<const f32x4_t*>(offs[buf] + 8 * v + 4 * hi);
                if (all) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sum[0] += __builtin_amdgcn_exp2f(fmaf(x0[4 * v + e], a.sl2, -o[e]));
                        sum[1] += __builtin_amdgcn_exp2f(fmaf(x1[4 * v + e], a.sl2, -o[e]));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t* m = bits[buf][8 * v + 4 * hi + e];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const bool sees = there[h] && (j[h] < 0 || (m[(j[h] >> 5) - w0] >> (j[h] & 31) & 1));
                            const float p = __builtin_amdgcn_exp2f(fmaf(h == 0 ? x0[4 * v + e] : x1[4 * v + e], a.sl2, -o[e]));
                            sum[h] += sees ? p : 0.f;
                        }
                    }
                }
            }
        }
        if (t + 1 < n_tiles) put(buf ^ 1);
    }
    const int64_t at = (static_cast<int64_t>(u.r) * a.hkv + u.g) * a.keys + 16 * static_cast<int64_t>(u.e0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float w = sum[h] + __shfl_xor(sum[h], 32);
        if (!there[h] || hi != 0) continue;
        if (j[h] < 0 && a.before) w = fmaf(a.decay, a.before[at + place[h]], w);
        a.out[at + place[h]] = w;
    }
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
    a.chunk = kManyChunk;
    if (few) {
        const int64_t even = static_cast<int64_t>(b.n_kv_blocks) * s.hkv / 768;
        a.chunk = static_cast<int32_t>(std::max<int64_t>(8, std::min<int64_t>(kFewChunk, (even + 7) / 8 * 8)));
    }
    a.n_chunks = (b.max_blocks + a.chunk - 1) / a.chunk;
    const int64_t direct = static_cast<int64_t>(a.n_chunks) * b.n_rows * s.hkv;
    const int64_t counted = (b.n_kv_blocks / a.chunk + static_cast<int64_t>(b.n_rows)) * s.hkv;
    a.search = direct > 4 * counted;
    const int64_t grid = a.search ? counted : direct;
    if (grid > INT32_MAX)
        return set_error(TKV_EINVAL, "tkv_key_weights: %lld workgroups are too many", static_cast<long long>(grid));
    const auto run = [&](auto kernel) { kernel<<<dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, st>>>(a); };
    if (s.d == 128)
        few ? run(weigh_few<128>) : run(weigh_many<128>);
    else
        few ? run(weigh_few<64>) : run(weigh_many<64>);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TKV_OK : set_error(TKV_EHIP, "tkv_key_weights launch: %s", hipGetErrorString(e));
}
