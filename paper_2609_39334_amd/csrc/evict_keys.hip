// Eviction from the paged cache (tkv_evict_keys): of each row and KV head the first keys, the last ones, and the heaviest of
// those between stay, `budget` in all, and move in path order to the blocks of the row's new table.
//
// Two launches.  choose: a workgroup a (row, head) finds the weight of the last key that stays by radix selection over the
// weights' bits (11, 11 and 10 of them, the counts in LDS), then lists the kept keys in path order; keys of equal weight
// stay from the lowest index on.  move: a wave a new block copies the kept K and V rows, and the weights.
//
// A call has to read the weights once and to read and write what is kept, 8 d bytes a key: large calls are bound by memory in
// move, small ones by the chain of choose's steps.  One row of 30,000 keys, 2,048 of which stay (28/4/128): choose 19 us on 4 CUs
// (6 to cut, 4 for the orders and the first counts, which a CU's own rate bounds), move 4.3.  64 rows of up to 6,144 keys, 1,024
// of which stay (12/2/128): 10.6 and 24 us.  32 rows of 2,000 to 12,000 keys, 2,000 of which stay (32/8/128, 535 MB): 14 and 107
// us, 4.9 TB/s in move, a large copy's rate being 5.2.  One kernel for both leaves too few workgroups for the copies: 48 us for
// the first, 48 against 43 for the second, 128 against 131 for the third (before reads went past the caches).  The orders of 32
// slots a thread in registers, unrolled, took 27 us for 1,000 keys (instruction fetches) against 8.5.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cstdint>

#include "internal.h"
#include "rows.h"

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef f32x4_t f32x4_u __attribute__((aligned(4)));  // rows start anywhere

constexpr int kChoose = 1024, kChooseWaves = kChoose / 64;
constexpr int kCached = 8192;   // entries whose lengths stay in LDS
constexpr int kBins = 2048;
constexpr int kListed = 2048;   // most slots of a bin that are listed (30,000 keys: 26 us a call, 28 without the list)
constexpr int kEarly = 4;       // slots of a thread, in fours, whose weights are on their way at once: 16,384 of a row (32,768: 0.4 us slower)
constexpr int kHeld = 32768;    // slots whose orders stay in LDS, 128 KB; others are read again for every pass
constexpr int kMove = 256, kMoveWaves = kMove / 64;
// The old rows are not read again, so they are read past the caches (64 rows of up to 6,144 keys, 1,024 of which stay, 12/2/128
// heads: 36 us a call, 43 through them); the new ones are next read by attention, and written past the caches only where they
// do not fit them (32 rows of eight heads, 2,000 keys each, 250 MiB: 127 us, 131 into them; those 64 rows 40 us).
constexpr int64_t kPast = 192 << 20;

struct Args {
    tkv_evict_batch b;
    int32_t num_blocks, hkv, new_max, per_row, held;  // blocks of the longest new table, workgroups that move it; slots whose orders stay in LDS
    const float* weights;
    float* out;
    int64_t keys;
    uint16_t *k, *v;
    int32_t *kept, *n_kept;
    bool past;  // the kept keys are written past the caches
};

// A slot's order, an unsigned number: the weights' own (NaN below all others, the two zeros equal), 0 where there is no key,
// kStays for a key that stays whatever its weight.
constexpr uint32_t kStays = 0xffffffffu;
__device__ __forceinline__ uint32_t order_of(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);  // (-0 + 0 is 0)
    return w != w ? 1 : u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}

__global__ __launch_bounds__(kChoose) void choose(Args a) {
    extern __shared__ u32x4_t held[];  // the slots' orders, four by four, of the first a.held of them
    __shared__ uint8_t cached[kCached];
    __shared__ uint32_t hist[kBins];
    __shared__ int part[kChooseWaves], tally[2][kChooseWaves], found[6], list[kListed];
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = blockIdx.x / a.hkv, g = blockIdx.x - r * a.hkv;
    const tkv::RowTable tab = tkv::row_table(a.b.kv_indptr, r, a.b.n_kv_blocks, a.b.max_blocks);
    const tkv::RowTable to = tkv::row_table(a.b.new_indptr, r, a.b.n_new_blocks, a.b.n_new_blocks);
    const int budget = a.b.budget[r];
    int32_t* kept = a.kept + (static_cast<int64_t>(r) * a.hkv + g) * a.b.max_budget;
    const float* weights = a.weights + (static_cast<int64_t>(r) * a.hkv + g) * a.keys;

    const int fresh = to.ok && tid < to.n ? a.b.new_blocks[to.first + tid] : -1;
    const int quads = 4 * tab.n, in_lds = min(quads, a.held / 4);
    const auto weights_of = [&](int q) { return *reinterpret_cast<const f32x4_u*>(weights + 4 * static_cast<int64_t>(q)); };
    f32x4_t early[kEarly];  // (asked for before anything is known of the path)
#pragma unroll
    for (int k = 0; k < kEarly; ++k) early[k] = tid + k * kChoose < quads ? weights_of(tid + k * kChoose) : f32x4_t{};
    for (int i = tid; i < kBins; i += kChoose) hist[i] = 0;

    // the path's length, and where its keys between the first and the last begin and end: a thread a run of entries
    bool ok = tab.ok && to.ok && budget >= 0 && budget <= a.b.max_budget;
    const int end = 16 * tab.n, sink = min(a.b.sink, budget), recent = min(a.b.recent, budget - sink);
    const auto look = [&](int e) {
        int id;
        return tkv::entry_len(a.b.kv_blocks, a.b.block_len, a.num_blocks, tab.first + e, id);
    };
    const auto len_of = [&](int e) { return e < kCached ? static_cast<int>(cached[e]) : look(e); };
    const int stretch = (tab.n + kChoose - 1) / kChoose, e0 = min(tid * stretch, tab.n), e1 = min(e0 + stretch, tab.n);
    int mine = 0, N;
#pragma unroll 2
    for (int e = e0; e < e1; ++e) {
        const int len = look(e);
        if (e < kCached) cached[e] = static_cast<uint8_t>(len);
        mine += len;
    }
    int number = tkv::group_before<kChooseWaves>(mine, N, part);
    for (int e = e0; e < e1; ++e) {
        const int len = len_of(e);
        if (sink >= number && sink < number + len) found[0] = 16 * e + (sink - number);
        if (N - recent >= number && N - recent < number + len) found[1] = 16 * e + (N - recent - number);
        number += len;
    }
    const int n = ok ? min(N, budget) : 0, need = (n + 15) / 16;
    // new blocks that are not of the pool
    int bad = need > to.n || (tid < need && static_cast<uint32_t>(fresh) >= static_cast<uint32_t>(a.num_blocks));
    for (int e = kChoose + tid; e < min(need, to.n); e += kChoose)
        if (static_cast<uint32_t>(a.b.new_blocks[to.first + e]) >= static_cast<uint32_t>(a.num_blocks)) bad = 1;
    if (__syncthreads_or(bad)) ok = false;
    const int n_out = ok ? n : 0;
    for (int i = n_out + tid; i < a.b.max_budget; i += kChoose) kept[i] = -1;
    if (g == 0 && tid == 0) a.n_kept[r] = ok ? n : -1;
    if (n_out == 0) return;
    const int lo = N <= budget ? end : found[0], hi = N <= budget || recent == 0 ? end : found[1];
    // the orders of slots 4 q .. 4 q + 3, of one entry
    const auto orders_of = [&](int q, f32x4_t w) {
        const int len = len_of(q >> 2), slot = 4 * q & 15;
        u32x4_t o;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = 4 * q + k;
            o[k] = i < lo || i >= hi ? kStays : order_of(w[k]);
            if (slot + k >= len) o[k] = 0;
        }
        return o;
    };
    const auto orders = [&](int q) { return q < in_lds ? held[q] : orders_of(q, weights_of(q)); };
    // equal weights are common: one addition where all lanes of a wave have the same bin
    const auto add = [&](uint32_t bin) {
        const uint32_t first = __builtin_amdgcn_readfirstlane(bin);
        const uint64_t all = __builtin_amdgcn_ballot_w64(true);
        if (__builtin_amdgcn_ballot_w64(bin != first) != 0)
            atomicAdd(hist + bin, 1u);
        else if (lane == __builtin_ctzll(all))
            atomicAdd(hist + bin, static_cast<uint32_t>(__builtin_popcountll(all)));
    };
    const auto fill = [&](int q, f32x4_t w) {
        const u32x4_t o = orders_of(q, w);
        if (q < in_lds) held[q] = o;
        const uint32_t first = __builtin_amdgcn_readfirstlane(o[0]) >> 21;
        const uint32_t apart = (o[0] >> 21 ^ first) | ((o[0] ^ o[1]) | (o[0] ^ o[2]) | (o[0] ^ o[3])) >> 21;
        if (first != 0 && __builtin_amdgcn_ballot_w64(apart != 0) == 0) {
            const uint64_t all = __builtin_amdgcn_ballot_w64(true);
            if (lane == __builtin_ctzll(all)) atomicAdd(hist + first, static_cast<uint32_t>(4 * __builtin_popcountll(all)));
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (o[k] != 0) atomicAdd(hist + (o[k] >> 21), 1u);
        }
    };
    for (int q = tid; q < quads; q += kEarly * kChoose) {
#pragma unroll
        for (int k = 0; k < kEarly; ++k) {
            const int mine = q + k * kChoose, later = mine + kEarly * kChoose;
            const f32x4_t w = early[k];
            if (later < quads) early[k] = weights_of(later);
            if (mine < quads) fill(mine, w);
        }
    }
    // The order of the last key that stays, 11, 11 and 10 bits at a time, and how many of that order do.  Where the first bin
    // that is not kept whole is small, its slots are listed as they are counted, and the rest goes by the list.
    const int run = (quads + 64 * kChooseWaves - 1) / (64 * kChooseWaves) * 64;  // a wave a run of slots, in fours
    const int from = min(wid * run, quads), until = min(from + run, quads);
    const auto order = [&](int i) { return i < 4 * in_lds ? reinterpret_cast<const uint32_t*>(held)[i] : orders(i >> 2)[i & 3]; };
    uint32_t last = 0;
    int left = n, n_listed = 0;
    bool listed = false;
    for (int low = 21;;) {
        __syncthreads();
        // the bin, counted from the largest, in which it lies
        const int most = low == 0 ? 0x3ff : 0x7ff, top = most - 2 * tid;
        const int h0 = top >= 0 ? hist[top] : 0, h1 = top >= 1 ? hist[top - 1] : 0;
        int total;
        const int above = tkv::group_before<kChooseWaves>(h0 + h1, total, part);
        if (above < left && left <= above + h0) found[2] = top, found[3] = left - above, found[4] = h0;
        if (above + h0 < left && left <= above + h0 + h1) found[2] = top - 1, found[3] = left - above - h0, found[4] = h1;
        if (tid == 0) found[5] = 0;
        __syncthreads();
        last |= static_cast<uint32_t>(found[2]) << low;
        left = found[3];
        if (low == 0) break;
        if (found[4] == left) {  // the whole bin stays: those of its lowest order as well
            last = max(last, 1u);
            break;
        }
        const int shift = low;
        low = low == 21 ? 10 : 0;
        const uint32_t mask = low == 0 ? 0x3ff : 0x7ff;
        for (int i = tid; i < kBins; i += kChoose) hist[i] = 0;
        if (low == 10) listed = found[4] <= kListed, n_listed = found[4];
        __syncthreads();
        if (low == 10 && listed) {
            const uint32_t least = max(last, 1u), most_of = last | 0x1fffff;
            int sures = 0;
            for (int base = from; base < until; base += 64) {
                const int q = base + lane;
                const u32x4_t o = q < until ? orders(q) : u32x4_t{0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    sures += __builtin_popcountll(__builtin_amdgcn_ballot_w64(o[k] > most_of));
                    if (o[k] - least <= most_of - least) {
                        list[atomicAdd(found + 5, 1)] = 4 * q + k;
                        atomicAdd(hist + (o[k] >> 10 & 0x7ff), 1u);
                    }
                }
            }
            if (lane == 0) tally[0][wid] = sures, tally[1][wid] = 0;
        } else if (listed) {
            for (int c = tid; c < n_listed; c += kChoose) {
                const uint32_t o = order(list[c]);
                if ((o ^ last) >> shift == 0) atomicAdd(hist + (o >> low & mask), 1u);
            }
        } else {
#pragma unroll 2
            for (int q = tid; q < quads; q += kChoose) {
                const u32x4_t o = orders(q);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (o[k] != 0 && ((o[k] ^ last) >> shift) == 0) add(o[k] >> low & mask);
            }
        }
    }

    // the kept ones in path order, counted first
    if (listed) {
        for (int c = tid; c < n_listed; c += kChoose) {
            const int i = list[c];
            const uint32_t o = order(i);
            if (o > last) atomicAdd(&tally[0][(i >> 2) / run], 1);
            if (o == last) atomicAdd(&tally[1][(i >> 2) / run], 1);
        }
    } else {
        int sures = 0, equals = 0;
        for (int base = from; base < until; base += 64) {
            const int q = base + lane;
            const u32x4_t o = q < until ? orders(q) : u32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sures += __builtin_popcountll(__builtin_amdgcn_ballot_w64(o[k] > last));
                equals += __builtin_popcountll(__builtin_amdgcn_ballot_w64(o[k] == last));
            }
        }
        if (lane == 0) tally[0][wid] = sures, tally[1][wid] = equals;
    }
    __syncthreads();
    int sures = 0, equals = 0;
    for (int x = 0; x < wid; ++x) sures += tally[0][x], equals += tally[1][x];
    // x and the lanes of m before this one
    const auto below = [](uint64_t m, int x) {
        return static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), x)));
    };
#pragma unroll 2
    for (int base = from; base < until; base += 64) {
        const int q = base + lane;
        const u32x4_t o = q < until ? orders(q) : u32x4_t{0, 0, 0, 0};
        uint64_t s[4], e[4];
        int at = sures, rank = equals;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            s[k] = __builtin_amdgcn_ballot_w64(o[k] > last), e[k] = __builtin_amdgcn_ballot_w64(o[k] == last);
            at = below(s[k], at);
            sures += __builtin_popcountll(s[k]);
        }
        if ((e[0] | e[1] | e[2] | e[3]) == 0) {
            at += min(rank, left);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (o[k] > last) kept[at++] = 4 * q + k;
            continue;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            rank = below(e[k], rank);
            equals += __builtin_popcountll(e[k]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (o[k] > last || (o[k] == last && rank < left)) kept[at + min(rank, left)] = 4 * q + k;
            at += o[k] > last, rank += o[k] == last;
        }
    }
}

template <int D>
__global__ __launch_bounds__(kMove) void move(Args a) {
    constexpr int CPR = D / 8, RPI = 64 / CPR, NI = 16 / RPI;  // 16-byte pieces a row, rows a load, loads a block
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    const int per_row = a.per_row;
    const int x = blockIdx.x % per_row, u = blockIdx.x / per_row;
    const int g = u % a.hkv, r = u / a.hkv;
    const int j = x * kMoveWaves + wid, n = a.n_kept[r] - 16 * j;
    if (n <= 0) return;
    // lane l holds the source of slot l % 16
    const int64_t head = static_cast<int64_t>(r) * a.hkv + g;
    const int i = a.kept[head * a.b.max_budget + 16 * j + min(lane & 15, n - 1)];
    if (lane < min(16, n)) a.out[head * a.keys + 16 * j + lane] = a.weights[head * a.keys + i];
    const int id = a.b.kv_blocks[a.b.kv_indptr[r] + (i >> 4)];
    const int64_t to = (static_cast<int64_t>(a.b.new_blocks[a.b.new_indptr[r] + j]) * a.hkv + g) * (16 * D);
    u32x4_t kx[NI], vx[NI];
#pragma unroll
    for (int s = 0; s < NI; ++s) {
        const int row = s * RPI + lane / CPR;
        const int64_t from = (static_cast<int64_t>(__shfl(id, row)) * a.hkv + g) * (16 * D) + (__shfl(i, row) & 15) * D + lane % CPR * 8;
        kx[s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(a.k + from));
        vx[s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(a.v + from));
    }
#pragma unroll
    for (int s = 0; s < NI; ++s) {
        const int row = s * RPI + lane / CPR;
        if (row >= n) continue;
        u32x4_t* kt = reinterpret_cast<u32x4_t*>(a.k + to + row * D + lane % CPR * 8);
        u32x4_t* vt = reinterpret_cast<u32x4_t*>(a.v + to + row * D + lane % CPR * 8);
        if (a.past) {
            asm volatile("");  // (the branches would be made one, and the stores ordinary ones)
            __builtin_nontemporal_store(kx[s], kt);
            __builtin_nontemporal_store(vx[s], vt);
            asm volatile("");
        } else {
            *kt = kx[s], *vt = vx[s];
        }
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
    a.per_row = (a.new_max + kMoveWaves - 1) / kMoveWaves | 1;  // (odd: a row's blocks would go to the same XCDs as the other rows')
    const int64_t moves = a.new_max > 0 ? rows * a.per_row : 0;
    if (rows > static_cast<int64_t>(UINT32_MAX) / kChoose || moves > static_cast<int64_t>(UINT32_MAX) / kMove)
        return set_error(TKV_EINVAL, "tkv_evict_keys: %lld workgroups are too many", static_cast<long long>(std::max(rows, moves)));
    a.past = rows * b.max_budget * s.d * 4 >= kPast;
    a.held = std::min(kHeld, 16 * b.max_blocks);
    choose<<<dim3(static_cast<unsigned>(rows)), dim3(kChoose), static_cast<size_t>(a.held) * 4, st>>>(a);
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
