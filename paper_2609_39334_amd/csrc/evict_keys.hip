// Eviction from the paged cache (tkv_evict_keys): of each row and KV head the first keys, the last ones, and the heaviest of
// those between stay, `budget` in all, and move in path order to the blocks of the row's new table.
//
// Two launches.  choose: a workgroup a (row, head) finds the weight of the last key that stays by radix selection over the
// weights' bits (11, 11 and 10 of them, the counts in LDS), then lists the kept keys in path order; keys of equal weight
// stay from the lowest index on.  move: a wave a new block copies the kept K and V rows.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cstdint>

#include "internal.h"
#include "rows.h"

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kChoose = 1024, kChooseWaves = kChoose / 64;
constexpr int kCached = 16384;  // entries whose lengths stay in LDS
constexpr int kBins = 2048;
constexpr int kMove = 256, kMoveWaves = kMove / 64;

struct Args {
    tkv_evict_batch b;
    int32_t num_blocks, hkv, new_max;  // blocks of the longest new table
    const float* weights;
    float* out;
    int64_t keys;
    uint16_t *k, *v;
    int32_t *kept, *n_kept;
};

// Unsigned numbers in the order of the weights: NaN below everything, the two zeros equal.
__device__ __forceinline__ uint32_t order_of(float w) {
    const uint32_t u = __float_as_uint(w);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
    if (u == 0x80000000u) return u;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kChoose) void choose(Args a) {
    __shared__ uint8_t cached[kCached];
    __shared__ uint32_t hist[kBins];
    __shared__ int part[kChooseWaves], part2[kChooseWaves], found[4];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const int r = blockIdx.x / a.hkv, g = blockIdx.x - r * a.hkv;
    const tkv::RowTable tab = tkv::row_table(a.b.kv_indptr, r, a.b.n_kv_blocks, a.b.max_blocks);
    const tkv::RowTable to = tkv::row_table(a.b.new_indptr, r, a.b.n_new_blocks, a.b.n_new_blocks);
    const int budget = a.b.budget[r];
    int32_t* kept = a.kept + (static_cast<int64_t>(r) * a.hkv + g) * a.b.max_budget;
    const float* w = a.weights + (static_cast<int64_t>(r) * a.hkv + g) * a.keys;
    float* out = a.out + (static_cast<int64_t>(r) * a.hkv + g) * a.keys;

    // the path's length, and where its keys between the first and the last begin and end
    bool ok = tab.ok && to.ok && budget >= 0 && budget <= a.b.max_budget;
    const int sink = min(a.b.sink, budget);
    int N = 0, lo = 0, hi = 16 * tab.n;
    for (int base = 0; ok && base < tab.n; base += kChoose) {
        const int e = base + tid;
        int id, len = 0, total;
        if (e < tab.n) len = tkv::entry_len(a.b.kv_blocks, a.b.block_len, a.num_blocks, tab.first + e, id);
        if (e < kCached) cached[e] = static_cast<uint8_t>(len);
        const int number = N + tkv::group_before<kChooseWaves>(len, total, part);
        if (sink >= number && sink < number + len) found[0] = 16 * e + (sink - number);
        N += total;
        __syncthreads();
    }
    const int n = ok ? min(N, budget) : 0;
    if (ok && N > budget && budget > 0) lo = found[0];
    // new blocks that are not of the pool
    {
        int bad = 0;
        for (int e = tid; e < (n + 15) / 16; e += kChoose)
            if (e >= to.n || static_cast<uint32_t>(a.b.new_blocks[to.first + e]) >= static_cast<uint32_t>(a.num_blocks)) bad = 1;
        int any;
        tkv::group_before<kChooseWaves>(bad, any, part);
        if (any) ok = false;
        __syncthreads();
    }
    const int n_out = ok ? n : 0;
    for (int i = n_out + tid; i < a.b.max_budget; i += kChoose) kept[i] = -1;
    if (g == 0 && tid == 0) a.n_kept[r] = ok ? n : -1;
    if (n_out == 0) return;

    const auto len_of = [&](int e) {
        int id;
        return e < kCached ? static_cast<int>(cached[e]) : tkv::entry_len(a.b.kv_blocks, a.b.block_len, a.num_blocks, tab.first + e, id);
    };
    uint32_t last = 0;  // the order of the last key that stays, and how many of that order do
    int equals = 0;
    if (N <= budget) {
        lo = hi;
    } else {
        const int recent = min(a.b.recent, budget - sink);
        int after = 0;
        for (int base = (tab.n - 1) / kChoose * kChoose; recent > 0 && base >= 0 && after < recent; base -= kChoose) {
            const int e = base + tid;
            int total;
            const int len = e < tab.n ? len_of(e) : 0;
            const int before = tkv::group_before<kChooseWaves>(len, total, part);
            const int behind = after + total - before - len;  // keys behind this entry
            if (behind < recent && recent <= behind + len) found[1] = 16 * e + (len - (recent - behind));
            after += total;
            __syncthreads();
        }
        if (recent > 0) hi = found[1];
        int left = budget - sink - recent;
        if (left == 0) {
            last = 0xffffffffu, equals = 0;  // (no weight has this order)
        } else {
            uint32_t high = 0;
            for (int pass = 0; pass < 3; ++pass) {
                const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
                for (int i = tid; i < kBins; i += kChoose) hist[i] = 0;
                __syncthreads();
                for (int i = lo + tid; i < hi; i += kChoose) {
                    if ((i & 15) >= len_of(i >> 4)) continue;
                    const uint32_t o = order_of(w[i]);
                    if (pass > 0 && (o ^ high) >> (shift + width) != 0) continue;
                    atomicAdd(hist + (o >> shift & ((1u << width) - 1)), 1u);
                }
                __syncthreads();
                // the bin, counted from the largest, in which the last one lies
                const int top = (1 << width) - 1 - 2 * tid;
                const int h0 = top >= 0 ? hist[top] : 0, h1 = top >= 1 ? hist[top - 1] : 0;
                int total;
                const int above = tkv::group_before<kChooseWaves>(h0 + h1, total, part);
                if (above < left && left <= above + h0) found[2] = top, found[3] = left - above;
                if (above + h0 < left && left <= above + h0 + h1) found[2] = top - 1, found[3] = left - above - h0;
                __syncthreads();
                high |= static_cast<uint32_t>(found[2]) << shift;
                left = found[3];
                __syncthreads();
            }
            last = high, equals = left;
        }
    }

    // the kept ones in path order: a wave a run of slots, counted first
    const int end = 16 * tab.n, run = (end + 64 * kChooseWaves - 1) / (64 * kChooseWaves) * 64;
    const int from = min(wid * run, end), until = min(from + run, end);
    const auto look = [&](int i, bool& sure, bool& equal, float& x) {
        const bool there = i < until && (i & 15) < len_of(i >> 4);
        x = there ? w[i] : 0.f;
        const bool between = i >= lo && i < hi;
        const uint32_t o = order_of(x);
        sure = there && (!between || o > last);
        equal = there && between && o == last;
    };
    int n_sure = 0, n_equal = 0;
    for (int i = from; i < until; i += 64) {
        bool sure, equal;
        float x;
        look(i + lane, sure, equal, x);
        n_sure += __builtin_popcountll(__builtin_amdgcn_ballot_w64(sure));
        n_equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(equal));
    }
    if (lane == 0) part[wid] = n_sure, part2[wid] = n_equal;
    __syncthreads();
    int sures = 0, same = 0;
    for (int x = 0; x < wid; ++x) sures += part[x], same += part2[x];
    for (int i = from; i < until; i += 64) {
        bool sure, equal;
        float x;
        look(i + lane, sure, equal, x);
        const uint64_t below = (uint64_t{1} << lane) - 1;
        const uint64_t se = __builtin_amdgcn_ballot_w64(equal), ss = __builtin_amdgcn_ballot_w64(sure);
        const int rank = same + __builtin_popcountll(se & below);
        const int at = sures + __builtin_popcountll(ss & below) + min(rank, equals);
        if (sure || (equal && rank < equals)) {
            kept[at] = i + lane;
            out[at] = x;
        }
        sures += __builtin_popcountll(ss), same += __builtin_popcountll(se);
    }
}

template <int D>
__global__ __launch_bounds__(kMove) void move(Args a) {
    constexpr int CPR = D / 8, RPI = 64 / CPR, NI = 16 / RPI;  // 16-byte pieces a row, rows a load, loads a block
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    const int per_row = (a.new_max + kMoveWaves - 1) / kMoveWaves;
    const int x = blockIdx.x % per_row, u = blockIdx.x / per_row;
    const int g = u % a.hkv, r = u / a.hkv;
    const int j = x * kMoveWaves + wid, n = a.n_kept[r] - 16 * j;
    if (n <= 0) return;
    // lane l holds the source of slot l % 16
    const int32_t* kept = a.kept + (static_cast<int64_t>(r) * a.hkv + g) * a.b.max_budget + 16 * j;
    const int i = kept[min(lane & 15, n - 1)];
    const int id = a.b.kv_blocks[a.b.kv_indptr[r] + (i >> 4)];
    const int64_t to = (static_cast<int64_t>(a.b.new_blocks[a.b.new_indptr[r] + j]) * a.hkv + g) * (16 * D);
    u32x4_t kx[NI], vx[NI];
#pragma unroll
    for (int s = 0; s < NI; ++s) {
        const int row = s * RPI + lane / CPR;
        const int64_t from = (static_cast<int64_t>(__shfl(id, row)) * a.hkv + g) * (16 * D) + (__shfl(i, row) & 15) * D + lane % CPR * 8;
        kx[s] = *reinterpret_cast<const u32x4_t*>(a.k + from);
        vx[s] = *reinterpret_cast<const u32x4_t*>(a.v + from);
    }
#pragma unroll
    for (int s = 0; s < NI; ++s) {
        const int row = s * RPI + lane / CPR;
        if (row >= n) continue;
        *reinterpret_cast<u32x4_t*>(a.k + to + row * D + lane % CPR * 8) = kx[s];
        *reinterpret_cast<u32x4_t*>(a.v + to + row * D + lane % CPR * 8) = vx[s];
    }
}

}  // namespace

int tkv::launch_evict_keys(const tkv_shape& s, const tkv_evict_batch& b, const float* weights, float* out, int64_t keys, void* k,
                           void* v, int32_t* kept, int32_t* n_kept, void* stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    Args a{};
    a.b = b;
    a.num_blocks = s.num_blocks, a.hkv = s.hkv;
    a.new_max = static_cast<int32_t>(std::min<int64_t>((static_cast<int64_t>(b.max_budget) + 15) / 16, b.n_new_blocks));
    a.weights = weights, a.out = out, a.keys = keys;
    a.k = static_cast<uint16_t*>(k), a.v = static_cast<uint16_t*>(v), a.kept = kept, a.n_kept = n_kept;
    const int64_t rows = static_cast<int64_t>(b.n_rows) * s.hkv;
    const int64_t moves = rows * ((a.new_max + kMoveWaves - 1) / kMoveWaves);
    if (rows > INT32_MAX || moves > INT32_MAX)
        return set_error(TKV_EINVAL, "tkv_evict_keys: %lld workgroups are too many", static_cast<long long>(std::max(rows, moves)));
    choose<<<dim3(static_cast<unsigned>(rows)), dim3(kChoose), 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(TKV_EHIP, "tkv_evict_keys launch: %s", hipGetErrorString(e));
    if (moves == 0) return TKV_OK;
    if (s.d == 128)
        move<128><<<dim3(static_cast<unsigned>(moves)), dim3(kMove), 0, st>>>(a);
    else
        move<64><<<dim3(static_cast<unsigned>(moves)), dim3(kMove), 0, st>>>(a);
    e = hipGetLastError();
    return e == hipSuccess ? TKV_OK : set_error(TKV_EHIP, "tkv_evict_keys launch (move): %s", hipGetErrorString(e));
}
