// The attention weight that a batch's queries give each key (tkv_key_weights): for key x of a row and KV head g
//   w'[x] = decay w[x] [x is context] + sum over the tokens i that see x of coef_i sum over the heads h of g of
//           exp(q_ih . k_x / sqrt(d) - lse_ih),
// with lse from the attention call before.  S = Q K^T runs on v_mfma_f32_32x32x16_bf16 with the queries as its rows, so that a
// lane holds one key's scores against 16 queries and their sum stays in the lane; K goes from the pool straight into the
// operand.  A key of a row and head belongs to one wave, whose order of additions is fixed: no atomics.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cstdint>

#include "internal.h"
#include "rows.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kChunk = 16;  // entries a workgroup

struct Args {
    tkv_draft_batch b;
    int32_t num_blocks, hq, hkv, G, n_chunks;
    float sl2, decay;  // log2(e) / sqrt(d)
    const uint16_t *q, *k;
    const float *lse, *coef, *before;
    float* out;
    int64_t keys;  // of a row and head in before and out
};

// Keys of the table behind entry `next`, exact below `most`, to all threads.
__device__ __forceinline__ int keys_behind(const Args& a, const tkv::RowTable& tab, int next, int most, int* part) {
    int after = 0;
    while (after < most && next < tab.n) {
        int id, total, len = 0;
        if (next + static_cast<int>(threadIdx.x) < tab.n)
            len = tkv::entry_len(a.b.kv_blocks, a.b.block_len, a.num_blocks, tab.first + next + threadIdx.x, id);
        tkv::group_before<kWaves>(len, total, part);
        __syncthreads();
        after += total;
        next += kThreads;
    }
    return after;
}

template <int D>
__global__ __launch_bounds__(kThreads) void weigh(Args a) {
    constexpr int KS = D / 16;
    __shared__ int2 list[kChunk];  // {id, 32 (first key's drafted number, at least -64) + length}
    __shared__ int part[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const int chunk = blockIdx.x % a.n_chunks, u = blockIdx.x / a.n_chunks;
    const int g = u % a.hkv, r = u / a.hkv;
    const tkv::RowTokens t = tkv::row_tokens(a.b, r);
    const tkv::RowTable tab = tkv::row_table(a.b.kv_indptr, r, a.b.n_kv_blocks, a.b.max_blocks);
    const int e0 = chunk * kChunk;
    if (!t.ok || !tab.ok || e0 >= tab.n) return;
    {
        const int after = keys_behind(a, tab, e0 + kChunk, t.L, part);
        int id = 0, len = 0, total;
        if (tid < kChunk && e0 + tid < tab.n)
            len = tkv::entry_len(a.b.kv_blocks, a.b.block_len, a.num_blocks, tab.first + e0 + tid, id);
        const int before = tkv::group_before<kWaves>(len, total, part);
        if (tid < kChunk) list[tid] = int2{id, 32 * max(t.L - (after + total - before), -64) + len};
        __syncthreads();
    }
    const int col = lane & 31, hi = lane >> 5;
    const int rows = t.L * a.G;
    for (int p = wid; p < kChunk / 2; p += kWaves) {
        const int2 d = list[2 * p + (col >> 4)];
        const int len = d.y & 31, slot = col & 15;
        const bool there = slot < len;
        if (__builtin_amdgcn_ballot_w64(there) == 0) continue;
        const int j = (d.y >> 5) + slot;  // this lane's key among the drafted ones (negative: context)
        const bool drafted = __builtin_amdgcn_ballot_w64(there && j >= 0) != 0;
        bf16x8_t kf[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[s] = bf16x8_t{};
        if (there) {
            const uint16_t* row = a.k + (static_cast<int64_t>(d.x) * a.hkv + g) * (16 * D) + slot * D + 8 * hi;
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[s] = *reinterpret_cast<const bf16x8_t*>(row + 16 * s);
        }
        float sum = 0.f;
        for (int t0 = 0; t0 < rows; t0 += 32) {
            const int qr = min(t0 + col, rows - 1), qi = qr / a.G;
            const uint16_t* qrow = a.q + (static_cast<int64_t>(t.q0 + qi) * a.hq + g * a.G + (qr - qi * a.G)) * D + 8 * hi;
            f32x16_t x{};
#pragma unroll
            for (int s = 0; s < KS; ++s)
                x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8_t*>(qrow + 16 * s), kf[s], x, 0, 0, 0);
            // x[4 u + e] is query row 8 u + 4 hi + e
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int row = t0 + 8 * (e >> 2) + 4 * hi + (e & 3);
                if (row >= rows) continue;
                const int i = row / a.G;
                const int64_t at = t.q0 + i;
                const float c = a.coef ? a.coef[at] : 1.f, z = a.lse[at * a.hq + g * a.G + (row - i * a.G)];
                bool sees = fabsf(z) < INFINITY;
                if (drafted && j >= 0) sees = sees && (a.b.mask[at * a.b.mask_words + (j >> 6)] >> (j & 63) & 1);
                if (sees && c > 0.f) sum += c * __builtin_amdgcn_exp2f(x[e] * a.sl2 - z * 1.4426950408889634f);
            }
        }
        sum += __shfl_xor(sum, 32);
        if (there && hi == 0) {
            const int64_t at = (static_cast<int64_t>(r) * a.hkv + g) * a.keys + 16 * static_cast<int64_t>(e0 + 2 * p + (col >> 4)) + slot;
            if (j < 0 && a.before) sum += a.decay * a.before[at];
            a.out[at] = sum;
        }
    }
}

}  // namespace

int tkv::launch_key_weights(const tkv_shape& s, const tkv_draft_batch& b, const void* q, const void* k, const float* lse,
                            const float* coef, float decay, const float* before, float* out, int64_t keys, void* stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    Args a{};
    a.b = b;
    a.num_blocks = s.num_blocks, a.hq = s.hq, a.hkv = s.hkv, a.G = s.hq / s.hkv;
    a.sl2 = 1.4426950408889634f / sqrtf(static_cast<float>(s.d));
    a.decay = decay;
    a.q = static_cast<const uint16_t*>(q), a.k = static_cast<const uint16_t*>(k);
    a.lse = lse, a.coef = coef, a.before = decay != 0.f ? before : nullptr, a.out = out, a.keys = keys;
    a.n_chunks = (b.max_blocks + kChunk - 1) / kChunk;
    const int64_t grid = static_cast<int64_t>(a.n_chunks) * b.n_rows * s.hkv;
    if (grid > INT32_MAX)
        return set_error(TKV_EINVAL, "tkv_key_weights: %lld workgroups are too many", static_cast<long long>(grid));
    if (s.d == 128)
        weigh<128><<<dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, st>>>(a);
    else
        weigh<64><<<dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TKV_OK : set_error(TKV_EHIP, "tkv_key_weights launch: %s", hipGetErrorString(e));
}
