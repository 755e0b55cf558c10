// Attention of drafted token trees over the paged pool (tkv_draft_verify).  A row is a path of N keys whose last L
// are its drafted tokens; token i sees the context and the drafted keys whose bits are set in its mask.
//
// A workgroup contracts one tile of a row's query rows (L tokens x the G heads of one KV head) against one chunk of
// the row's blocks, in transposed products so that each lane keeps one query row throughout:
//   S^T = K Q^T,  O^T += V^T P^T   on v_mfma_f32_32x32x16_bf16, 32 query rows a wave,
// with an online softmax between them in fp32, whose base moves only when a row's maximum exceeds it by more than
// 2^8 in probability scale.  P is rounded to bf16 for the second product (2^-8 of each term at most, as in the other
// attention kernels here: the matrix instructions take no wider operands at that rate); the denominator sums it
// unrounded, so that lse has the precision of fp32.
//
// K and V go from the pool straight to LDS (buffer_load ... lds), double-buffered.  Which blocks these are is
// device data: the workgroup first reads its chunk's table entries and lengths, drops what is no block of the pool,
// and counts the keys from the row's end, which tells each block's place among the drafted tokens.  Stages of context
// alone run first, without looking at masks; in the others V is cleared of what is not finite, so that a hidden key may
// hold anything (under 1% of the time of the cases below), and what was cleared is added to the rows that see it.
//
// What bounds it (MI355X).  Single tokens: memory, 198 MB of keys (64 rows of 12/2/128 heads under 300 to 6,144 keys) in
// 42 us, 4.7 TB/s, and 4.6 us of merge; where the last-level cache holds the keys from the call before, 34 us.  Trees (with
// their keys in the cache; 32 rows take 4 us more without): the chain of a stage (K from LDS, MFMAs, exponentials, V, MFMAs) with two
// waves a SIMD.  8 rows of 64 to 150 tokens of 32/8/128 heads under 2,000 to 12,000 keys take 176 us, 610 TFLOP/s of seen
// keys; without the stages' loads 163, with the loads alone 98.  32 rows of 4 to 32 tokens, 28/4/128: 63 us, 57 and 41;
// 32 tokens under 30,000 keys 33 us, 33 and 23.  A unit costs 7 us beside its stages (its row, its table, the first
// stage, the partial result), a stage 1.4 to 2 us.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "internal.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void* lds_void_ptr;

constexpr int kThreads = 256;      // four waves
constexpr int kMaxChunk = 256;     // blocks of a chunk: one table entry a thread
constexpr uint32_t kNaNBits = 0x7fc00000u;

struct Args {
    tkv_draft_batch b;
    int32_t num_blocks, hq, hkv, G;
    int32_t chunk, n_chunks, n_tiles;  // most blocks of a chunk, chunks of the longest row, tiles of the widest row
    float sl2;                         // log2(e) / sqrt(d)
    const uint16_t *q, *k, *v;
    uint16_t* o;
    float *lse, *po, *plse;            // plse in units of log2
};

__device__ __forceinline__ f32x16_t mfma(bf16x8_t a, bf16x8_t b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{lo, hi}, bf16x2_t));
}

// Stage rows are D bf16, unpadded, their 16-byte chunks XOR-swizzled by row so that the operand reads below (K: 32
// rows of one chunk; V transposed: 4 rows of 64 bytes per 32 lanes) meet no bank conflict.
template <int D>
__device__ __forceinline__ int swz_k(int r) {
    return D == 128 ? r & 15 : (r >> 1) & 7;
}
template <int D>
__device__ __forceinline__ int swz_v(int r) {
    return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1);
}

// This wave's NB / 4 blocks of a stage into LDS, 1 KB an instruction, through buffer descriptors that span one block.
// Rows past a block's length read its last row.
template <int D, int R, int NB>
__device__ __forceinline__ void fetch_part(const uint16_t* __restrict__ kpool, const uint16_t* __restrict__ vpool, int2 d,
                                           size_t blk_stride, size_t kvh_off, int wid, int lane, uint8_t* kd, uint8_t* vd) {
    constexpr int CPR = D / 8, RPI = 64 / CPR;  // 16-byte chunks a row, rows an instruction
    constexpr int kRsrcWord3 = 0x00020000;      // raw buffer, 32-bit data format
#pragma unroll
    for (int x = 0; x < NB / 4; ++x) {
        const int j = wid * (NB / 4) + x;
        const size_t boff = static_cast<size_t>(__builtin_amdgcn_readlane(d.x, j)) * blk_stride + kvh_off;
        const int last = (__builtin_amdgcn_readlane(d.y, j) & 31) - 1;
        const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(kpool + boff), 0, 32 * D, kRsrcWord3);
        const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(vpool + boff), 0, 32 * D, kRsrcWord3);
#pragma unroll
        for (int i = 0; i < 16 / RPI; ++i) {
            const int r = i * RPI + lane / CPR;
            const int row = min(r, last) * D * 2;
            const int at = j * 32 * D + i * 1024;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_void_ptr)(kd + at), 16, row + (((lane % CPR) ^ swz_k<D>(r)) * 16), 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_void_ptr)(vd + at), 16, row + (((lane % CPR) ^ swz_v<D>(r)) * 16), 0, 0, 0);
        }
    }
}

// A barrier over what is in LDS, loads on their way left alone.
__device__ __forceinline__ void local_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
__device__ __forceinline__ void stage_barrier() {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    local_barrier();
}

// This wave's block of a stage of V in LDS: what is not finite becomes 0; returns whether anything was.  (A key that a row
// does not see has weight 0 there, and 0 times infinity or NaN would be NaN.)
template <int D>
__device__ __forceinline__ bool clear_block(uint8_t* blk, int lane) {
    constexpr int N = D / 32;  // 16-byte pieces a lane
    uint4 x[N];
    u16x2_t most{0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = *reinterpret_cast<const uint4*>(blk + (i * 64 + lane) * 16);
        const uint32_t* w = &x[i].x;
#pragma unroll
        for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2_t, w[e] & 0x7fff7fffu));
    }
    if (__builtin_amdgcn_ballot_w64(most.x >= 0x7f80 || most.y >= 0x7f80) == 0) return false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t* w = &x[i].x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool hi = (w[e] & 0x7f800000u) == 0x7f800000u, lo = (w[e] & 0x7f80u) == 0x7f80u;
            w[e] = (hi ? 0u : w[e] & 0xffff0000u) | (lo ? 0u : w[e] & 0xffffu);
        }
        *reinterpret_cast<uint4*>(blk + (i * 64 + lane) * 16) = x[i];
    }
    return true;
}

// A row of the batch as the device arrays give it.
struct Row {
    int q0, L;         // its query tokens
    int kv0, n_blk;    // its table
    bool tokens, table;  // whether they are inside the arrays
    int n_chunks, chunk; // chunks of near-equal length, blocks a chunk (one chunk at least)
};
__device__ __forceinline__ Row row_of(const Args& a, int r) {
    const tkv_draft_batch& b = a.b;
    Row w;
    w.q0 = b.q_indptr[r];
    w.L = b.q_indptr[r + 1] - w.q0;
    w.kv0 = b.kv_indptr[r];
    w.n_blk = b.kv_indptr[r + 1] - w.kv0;
    w.tokens = w.q0 >= 0 && w.q0 <= b.n_qtok && w.L >= 1 && w.L <= b.max_q && w.L <= b.n_qtok - w.q0;
    w.table = w.kv0 >= 0 && w.kv0 <= b.n_kv_blocks && w.n_blk >= 0 && w.n_blk <= b.max_blocks && w.n_blk <= b.n_kv_blocks - w.kv0;
    w.n_chunks = w.table && w.n_blk > 0 ? (w.n_blk + a.chunk - 1) / a.chunk : 1;
    w.chunk = w.table ? ((w.n_blk + w.n_chunks - 1) / w.n_chunks + 3) & ~3 : 0;  // whole stages (a.chunk is a multiple of four)
    if (w.n_chunks > 1) w.n_chunks = (w.n_blk + w.chunk - 1) / w.chunk;
    return w;
}

// Length of table entry i, 0 if it is no block of the pool.
__device__ __forceinline__ int entry(const Args& a, int i, int& id) {
    id = a.b.kv_blocks[i];
    if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(a.num_blocks)) return 0;
    const int len = a.b.block_len[id];
    return len >= 1 && len <= tkv::kBlock ? len : 0;
}

__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Which of a block's keys this token sees, as 16 bits: key x is drafted token d0 + x (context below 0).
__device__ __forceinline__ uint32_t seen(const uint64_t* __restrict__ m, int words, int d0, int len) {
    uint64_t v = ~uint64_t{0};
    if (d0 >= 0) {
        const int w = d0 >> 6, s = d0 & 63;
        v = m[w] >> s;
        if (s > 48 && w + 1 < words) v |= m[w + 1] << (64 - s);
    } else if (d0 + len > 0) {
        v = (m[0] << -d0) | ((uint64_t{1} << -d0) - 1);
    }
    return static_cast<uint32_t>(v) & ((1u << len) - 1);
}

// Those values for the rows that see them, added as they are in the pool (a weight would not change what they make of a sum;
// a row that sees a key whose weight rounds to 0 gets them too).  row: the block's first row of this KV head; bits: the
// keys that this lane's row sees.
template <int D>
__device__ __forceinline__ void add_not_finite(f32x16_t (&acc)[D / 32], const uint16_t* __restrict__ row, uint32_t bits, int hi) {
#pragma unroll 1
    for (int key = 0; key < tkv::kBlock; ++key, row += D) {
        if (!(bits >> key & 1)) continue;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint2 x = *reinterpret_cast<const uint2*>(row + 32 * dt + 8 * u + 4 * hi);
                const uint32_t w[4] = {x.x << 16, x.x & 0xffff0000u, x.y << 16, x.y & 0xffff0000u};
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[dt][4 * u + e] += __uint_as_float((w[e] & 0x7f800000u) == 0x7f800000u ? w[e] : 0u);
            }
    }
}

// One tile of a row against one chunk: R waves of 32 query rows times NG groups of keys, NB blocks a stage.
template <int D, int R>
__device__ __forceinline__ void draft_tile(const Args& a, const Row& w, int chunk, int kvh, int tile) {
    constexpr int NG = 4 / R, NB = 4, BG = NB / NG;  // BG: blocks of a group's part of a stage
    constexpr int RB = 2 * D, kStage = NB * 16 * RB;
    static_assert(BG % 2 == 0, "32 keys an MFMA");
    __shared__ __attribute__((aligned(16))) uint8_t k0[kStage], v0[kStage], k1[kStage], v1[kStage];
    __shared__ int2 list[kMaxChunk];     // the chunk's blocks: {id, 32 (first key's drafted number) + length}
    __shared__ int wsum[4][4];
    __shared__ int odd[NB];              // blocks of the stage whose V was cleared of something
    __shared__ float xml[NG > 1 ? (NG - 1) * R * 128 : 1];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wave = wid % R, grp = wid / R;

    const int c0 = chunk * w.chunk;

    // this lane's query row
    const int col = lane & 31, hi = lane >> 5;
    const int qrow = tile * 32 * R + 32 * wave + col;
    const bool live = qrow < w.L * a.G;
    const int i = live ? qrow / a.G : w.L - 1;
    const int h = kvh * a.G + (live ? qrow - i * a.G : 0);
    const size_t orow = static_cast<size_t>(w.q0 + i) * a.hq + h;
    if (!w.table) {
        if (live && grp == 0) {
            for (int c = 8 * hi; c < D; c += 16) *reinterpret_cast<uint4*>(a.o + orow * D + c) = uint4{0, 0, 0, 0};
            if (a.lse && hi == 0) reinterpret_cast<uint32_t*>(a.lse)[orow] = kNaNBits;
        }
        return;
    }
    bf16x8_t qf[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
        qf[ks] = *reinterpret_cast<const bf16x8_t*>(a.q + orow * D + hi * 8 + ks * 16);
    const uint64_t* mask = a.b.mask + static_cast<size_t>(w.q0 + i) * a.b.mask_words;
    const bool hides = w.L > 1 || (a.b.mask[static_cast<size_t>(w.q0) * a.b.mask_words] & 1) == 0;  // (a lone token sees itself)

    // the chunk's blocks, and how many keys of the row follow it (exact below L)
    int nb, before_draft;  // blocks, and those of them that hold no drafted key (the first)
    {
        const int n = min(w.chunk, w.n_blk - c0);
        int id = 0, len = 0, after = 0, later;
        if (tid < n) len = entry(a, w.kv0 + c0 + tid, id);
        int next = c0 + n;
        if (next + tid < w.n_blk && tid < w.L) after = entry(a, w.kv0 + next + tid, later);
        next += min(kThreads, w.L);
        int incl = len;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(incl, o);
            if (lane >= o) incl += u;
        }
        const uint64_t has = __builtin_amdgcn_ballot_w64(len > 0);
        after = wave_sum(after);
        if (lane == 63) wsum[0][wid] = incl;
        if (lane == 0) wsum[1][wid] = __builtin_popcountll(has), wsum[2][wid] = after;
        __syncthreads();
        int before = 0, at = 0, total = 0;
        nb = 0, after = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            before += x < wid ? wsum[0][x] : 0;
            at += x < wid ? wsum[1][x] : 0;
            total += wsum[0][x];
            nb += wsum[1][x];
            after += wsum[2][x];
        }
        while (after < w.L && next < w.n_blk) {  // many entries that are no blocks, or more drafted tokens than threads
            int more = next + tid < w.n_blk ? entry(a, w.kv0 + next + tid, later) : 0;
            next += kThreads;
            more = wave_sum(more);
            __syncthreads();
            if (lane == 0) wsum[2][wid] = more;
            __syncthreads();
            after += wsum[2][0] + wsum[2][1] + wsum[2][2] + wsum[2][3];
        }
        const int d0 = w.L - (after + total - (before + incl - len));  // drafted number of this block's first key
        if (len > 0) list[at + __builtin_popcountll(has & ((uint64_t{1} << lane) - 1))] = int2{id, 32 * max(d0, -64) + len};
        const uint64_t context = __builtin_amdgcn_ballot_w64(len > 0 && d0 <= -len);
        if (lane == 0) wsum[3][wid] = __builtin_popcountll(context);
        __syncthreads();
        before_draft = wsum[3][0] + wsum[3][1] + wsum[3][2] + wsum[3][3];
    }
    const int n_stages = (nb + NB - 1) / NB;
    const size_t blk_stride = static_cast<size_t>(a.hkv) * (16 * D), kvh_off = static_cast<size_t>(kvh) * (16 * D);

    // Swizzled read offsets.  K, A operand of S^T: lane (col, hi) reads row col of a block pair, chunk 2 ks + hi.
    // V, transposed: 16 lanes (dims half) read rows 4 hi .. 4 hi + 3 of a block, then 8 rows further.
    const int koff = col * RB + 16 * (hi ^ swz_k<D>(col));
    const int vj = lane & 15, vrow = 4 * hi + (vj >> 2);
    const int voff = vrow * RB + 16 * ((2 * ((lane >> 4) & 1) + ((vj & 3) >> 1)) ^ swz_v<D>(vrow)) + 8 * (vj & 1);

    // lane l holds block NB s + l % NB of stage s (the last block past the end)
    auto stage_desc = [&](int st) { return list[min(NB * st + lane % NB, nb - 1)]; };
    auto fetch = [&](int2 d, uint8_t* kd, uint8_t* vd) {
        fetch_part<D, R, NB>(a.k, a.v, d, blk_stride, kvh_off, wid, lane, kd, vd);
    };
    f32x16_t acc[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) acc[dt] = f32x16_t{};
    float m = -INFINITY, l = 0.f;
    const bool wave_live = __builtin_amdgcn_ballot_w64(live) != 0;
    int2 dcur{}, dnxt{};
    if (nb > 0) {
        dcur = stage_desc(0);
        fetch(dcur, k0, v0);
        dnxt = stage_desc(1);
    }
    auto stage = [&](auto drafted, int st, const uint8_t* ks, uint8_t* vs, uint8_t* kn, uint8_t* vn) {
        constexpr bool kDrafted = decltype(drafted)::value;
        stage_barrier();
        if (st + 1 < n_stages) fetch(dnxt, kn, vn);
        const int2 dthis = dcur;
        dcur = dnxt;
        dnxt = stage_desc(st + 2);
        if (kDrafted && hides) {
            const bool some = clear_block<D>(vs + wid * 16 * RB, lane);
            if (lane == 0) odd[wid] = some;
            local_barrier();
        }
        const int first = NB * st + BG * grp;
        if (!wave_live || first >= nb) return;
        constexpr int P = BG / 2;
        f32x16_t sc[P];
#pragma unroll
        for (int p = 0; p < P; ++p) sc[p] = f32x16_t{};
        bf16x8_t kf[D / 16][P];
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
            for (int p = 0; p < P; ++p)
                kf[kk][p] = *reinterpret_cast<const bf16x8_t*>(ks + (grp * BG + 2 * p) * 16 * RB + (koff ^ (32 * kk)));
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
            for (int p = 0; p < P; ++p) sc[p] = mfma(kf[kk][p], qf[kk], sc[p]);
        // K reads up to eight operands ahead of the MFMAs that use them
        constexpr int kReads = D / 16 * P, kAhead = kReads < 8 ? kReads : 8;
        __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
        for (int kk = 0; kk < (kReads - kAhead) / 4; ++kk) {
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
        // sc[p][8 b + 4 u + x] is key 8 u + 4 hi + x of block 2 p + b of the group's part.  One uniform decision: mask
        // where a block is partial, absent or holds drafted keys.
        int blk[BG];
        bool mixed = first + BG > nb;
#pragma unroll
        for (int j = 0; j < BG; ++j) {
            blk[j] = __builtin_amdgcn_readlane(dthis.y, BG * grp + j);
            mixed = mixed || (blk[j] & 31) != 16 || (kDrafted && (blk[j] >> 5) > -16);
        }
        if (mixed) {
            asm volatile("");  // (a branch, not selects in every stage)
#pragma unroll
            for (int j = 0; j < BG; ++j) {
                const int len = first + j < nb ? blk[j] & 31 : 0;
                const uint32_t bits = (kDrafted ? seen(mask, a.b.mask_words, blk[j] >> 5, len) : (1u << len) - 1) >> (4 * hi);
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    if (!((bits >> (8 * (x >> 2) + (x & 3))) & 1)) sc[j >> 1][8 * (j & 1) + x] = -INFINITY;
            }
        }
        {
            constexpr float kSlack = 8.f;
            float mx = -INFINITY;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int x = 0; x < 16; x += 2) mx = fmaxf(mx, fmaxf(sc[p][x], sc[p][x + 1]));
            if (__builtin_amdgcn_ballot_w64(mx > m + kSlack / a.sl2) != 0) {  // false for mx = -inf
                const auto e = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                const float m_new = fmaxf(m, fmaxf(__uint_as_float(e[0]), __uint_as_float(e[1])));
                const float alpha = m == m_new ? 1.f : __builtin_amdgcn_exp2f((m - m_new) * a.sl2);
                l *= alpha;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) acc[dt] *= alpha;
                m = m_new;
            }
        }
        const float msc = m == -INFINITY ? 0.f : m * a.sl2;
#pragma unroll
        for (int j = 0; j < BG; ++j) {
            float pr[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) pr[x] = __builtin_amdgcn_exp2f(fmaf(sc[j >> 1][8 * (j & 1) + x], a.sl2, -msc));
            const uint4 pk{pack_bf16x2(pr[0], pr[1]), pack_bf16x2(pr[2], pr[3]), pack_bf16x2(pr[4], pr[5]),
                           pack_bf16x2(pr[6], pr[7])};
            l += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
            const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, pk);
            const uint8_t* vr = vs + (grp * BG + j) * 16 * RB;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) {
                const int off = voff ^ (64 * dt);
                const s16x4_t va = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4_t*)(const_cast<uint8_t*>(vr + off)));
                const s16x4_t vb = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4_t*)(const_cast<uint8_t*>(vr + 8 * RB + off)));
                acc[dt] = mfma(__builtin_bit_cast(bf16x8_t, __builtin_shufflevector(va, vb, 0, 1, 2, 3, 4, 5, 6, 7)), pb, acc[dt]);
            }
        }
        if (kDrafted && hides) {
            int some = 0;
#pragma unroll
            for (int j = 0; j < BG; ++j) some |= odd[BG * grp + j] << j;
            some = __builtin_amdgcn_readfirstlane(some);
            for (int j = 0; some != 0; ++j, some >>= 1) {
                if (!(some & 1) || first + j >= nb) continue;
                const int at = __builtin_amdgcn_readlane(dthis.y, BG * grp + j);
                add_not_finite<D>(acc, a.v + static_cast<size_t>(__builtin_amdgcn_readlane(dthis.x, BG * grp + j)) * blk_stride + kvh_off,
                                  seen(mask, a.b.mask_words, at >> 5, at & 31), hi);
            }
        }
    };
    // the stages of context alone, in pairs, then the rest
    int st = 0;
    for (const int end = before_draft / NB; st + 1 < end; st += 2) {
        stage(std::false_type{}, st, k0, v0, k1, v1);
        stage(std::false_type{}, st + 1, k1, v1, k0, v0);
    }
    for (; st < n_stages; st += 2) {
        stage(std::true_type{}, st, k0, v0, k1, v1);
        if (st + 1 < n_stages) stage(std::true_type{}, st + 1, k1, v1, k0, v0);
    }
    if constexpr (NG > 1) {
        // the other groups' results over their keys join the first's through LDS, 32 x D fp32 a wave
        constexpr int kPer = kStage / (32 * D * 4);  // results an array holds
        static_assert(kPer >= 1 && (NG - 1) * R <= 4 * kPer, "the results fit the stage buffers");
        auto slot = [&](int x) {
            uint8_t* s = x < kPer ? k0 : x < 2 * kPer ? v0 : x < 3 * kPer ? k1 : v1;
            return reinterpret_cast<float*>(s + (x % kPer) * (32 * D * 4)) + lane * 4;
        };
        __syncthreads();
        if (grp > 0) {
            const int x = (grp - 1) * R + wave;
            float* xa = slot(x);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    *reinterpret_cast<f32x4_t*>(xa + (4 * dt + u) * 256) =
                        f32x4_t{acc[dt][4 * u], acc[dt][4 * u + 1], acc[dt][4 * u + 2], acc[dt][4 * u + 3]};
            xml[x * 128 + lane] = m;
            xml[x * 128 + 64 + lane] = l;
        }
        __syncthreads();
        if (grp > 0) return;
        float mt = m;
#pragma unroll
        for (int y = 0; y < NG - 1; ++y) mt = fmaxf(mt, xml[(y * R + wave) * 128 + lane]);
        const float a0 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mt) * a.sl2);
        l *= a0;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) acc[dt] *= a0;
#pragma unroll 1
        for (int y = 0; y < NG - 1; ++y) {
            const int x = y * R + wave;
            const float my = xml[x * 128 + lane];
            const float ay = my == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((my - mt) * a.sl2);
            l = fmaf(xml[x * 128 + 64 + lane], ay, l);
            const float* xa = slot(x);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const f32x4_t b = *reinterpret_cast<const f32x4_t*>(xa + (4 * dt + u) * 256);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[dt][4 * u + e] = fmaf(b[e], ay, acc[dt][4 * u + e]);
                }
        }
        m = mt;
    }
    const float sum = l + __shfl_xor(l, 32);
    if (!live) return;
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const float lse2 = sum > 0.f ? m * a.sl2 + log2f(sum) : -INFINITY;
    if (w.n_chunks == 1) {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                *reinterpret_cast<uint2*>(a.o + orow * D + 32 * dt + 8 * u + 4 * hi) =
                    uint2{pack_bf16x2(acc[dt][4 * u] * inv, acc[dt][4 * u + 1] * inv),
                          pack_bf16x2(acc[dt][4 * u + 2] * inv, acc[dt][4 * u + 3] * inv)};
        if (a.lse && hi == 0) a.lse[orow] = lse2 * 0.6931471805599453f;
    } else {
        const size_t prow = static_cast<size_t>(chunk) * a.b.n_qtok * a.hq + orow;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                *reinterpret_cast<f32x4_t*>(a.po + prow * D + 32 * dt + 8 * u + 4 * hi) =
                    f32x4_t{acc[dt][4 * u] * inv, acc[dt][4 * u + 1] * inv, acc[dt][4 * u + 2] * inv, acc[dt][4 * u + 3] * inv};
        if (hi == 0) a.plse[prow] = lse2;
    }
}

// A workgroup a unit: a row's chunk, KV head and tile.  Which units there are is device data: every workgroup counts
// the rows' units up to its own, one row a thread, so that no slot of the chip is held by a chunk or tile that a
// shorter row lacks (32 rows of 4 to 32 tokens of 28/4/128 heads under 500 to 6,144 keys: 64 us, 90 with a grid over
// the maxima).
// Units of one (row, chunk, KV head) read the same keys and follow each other, in runs on one XCD as long as the widest row
// has tiles; where rows differ in width a run may end among them, and the rest reads the keys on the next XCD.
template <int D, int R>
__global__ __launch_bounds__(kThreads, 2) void draft_attn(Args a) {
    __shared__ int sums[4], found[4];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const int seq = blockIdx.x >> 3, run = a.n_tiles;
    const int unit = (seq / run) * (8 * run) + (blockIdx.x & 7) * run + seq % run;
    if (tid == 0) found[0] = -1;
    int64_t before = 0;
    for (int r0 = 0; r0 < a.b.n_rows && before <= unit; r0 += kThreads) {
        int mine = 0, tiles = 0;
        if (r0 + tid < a.b.n_rows) {
            const Row w = row_of(a, r0 + tid);
            if (w.tokens) tiles = (w.L * a.G + 32 * R - 1) / (32 * R), mine = w.n_chunks * a.hkv * tiles;
        }
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(incl, o);
            if (lane >= o) incl += u;
        }
        __syncthreads();
        if (lane == 63) sums[wid] = incl;
        __syncthreads();
        int64_t at = before + incl - mine;
        for (int x = 0; x < 4; ++x) {
            if (x < wid) at += sums[x];
            before += sums[x];
        }
        if (unit >= at && unit < at + mine) found[0] = r0 + tid, found[1] = static_cast<int>(unit - at), found[2] = tiles;
    }
    __syncthreads();
    const int r = __builtin_amdgcn_readfirstlane(found[0]), local = __builtin_amdgcn_readfirstlane(found[1]);
    const int tiles = __builtin_amdgcn_readfirstlane(found[2]);
    if (r < 0) return;
    const int g = local / tiles;
    draft_tile<D, R>(a, row_of(a, r), g / a.hkv, g % a.hkv, local - g * tiles);
}

// o = sum_c 2^(lse_c - M) o_c / sum_c 2^(lse_c - M) over a row's chunks: P threads share the chunks of four dims of a
// (token, head), and meet through LDS.
template <int D, int P>
__global__ __launch_bounds__(kThreads) void draft_merge(Args a, int per_row) {
    constexpr int C = D / 4, H = kThreads / (C * P);  // (token, head) rows a workgroup
    __shared__ f32x4_t part[P > 1 ? P : 1][H][C];
    __shared__ float weight[P][H], base[P][H];
    const int r = blockIdx.x / per_row, first = (blockIdx.x - r * per_row) * H;
    const Row w = row_of(a, r);
    if (!w.tokens || w.n_chunks == 1) return;
    const int c = threadIdx.x % C, h = threadIdx.x / C % H, p = threadIdx.x / (C * H);
    const bool live = first + h < w.L * a.hq;
    const size_t orow = static_cast<size_t>(w.q0) * a.hq + min(first + h, w.L * a.hq - 1), step = static_cast<size_t>(a.b.n_qtok) * a.hq;
    const int n = w.n_chunks;
    // eight chunks' results in flight, over a running maximum
    constexpr int U = 8;
    float top = -INFINITY, z = 0.f;
    f32x4_t s{0.f, 0.f, 0.f, 0.f};
    for (int j0 = p; j0 < n; j0 += U * P) {
        float l[U];
        f32x4_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t at = min(j0 + u * P, n - 1) * step + orow;
            l[u] = a.plse[at];
            v[u] = *reinterpret_cast<const f32x4_t*>(a.po + at * D + 4 * c);
        }
        float now = top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j0 + u * P >= n) l[u] = -INFINITY;
            now = fmaxf(now, l[u]);
        }
        if (now == -INFINITY) continue;
        const float keep = __builtin_amdgcn_exp2f(top - now);
        z *= keep;
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] *= keep;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float e = __builtin_amdgcn_exp2f(l[u] - now);
            z += e;
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] = fmaf(e, v[u][k], s[k]);
        }
        top = now;
    }
    if constexpr (P > 1) {
        part[p][h][c] = s;
        if (c == 0) weight[p][h] = z, base[p][h] = top;
        __syncthreads();
        if (p > 0) return;
        float now = top;
#pragma unroll
        for (int q = 1; q < P; ++q) now = fmaxf(now, base[q][h]);
        if (now > -INFINITY) {
            const float keep = __builtin_amdgcn_exp2f(top - now);
            z *= keep;
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] *= keep;
#pragma unroll
            for (int q = 1; q < P; ++q) {
                const float e = __builtin_amdgcn_exp2f(base[q][h] - now);
                z = fmaf(e, weight[q][h], z);
#pragma unroll
                for (int k = 0; k < 4; ++k) s[k] = fmaf(e, part[q][h][c][k], s[k]);
            }
            top = now;
        }
    }
    if (!live) return;
    const float inv = z > 0.f ? 1.f / z : 0.f;
    *reinterpret_cast<uint2*>(a.o + orow * D + 4 * c) = uint2{pack_bf16x2(s[0] * inv, s[1] * inv), pack_bf16x2(s[2] * inv, s[3] * inv)};
    if (a.lse && c == 0) a.lse[orow] = z > 0.f ? (top + log2f(z)) * 0.6931471805599453f : -INFINITY;
}

int launched(const char* fn) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TKV_OK : tkv::set_error(TKV_EHIP, "%s launch: %s", fn, hipGetErrorString(e));
}

template <int D, int R>
int launch(const Args& a, hipStream_t st) {
    // as many units as every row having the longest table, or as the tables' blocks can make
    const int64_t heads = static_cast<int64_t>(a.hkv) * a.n_tiles;
    const int64_t most = static_cast<int64_t>(a.n_chunks) * a.b.n_rows * heads;
    const int64_t grid = std::min(most, (a.b.n_kv_blocks / a.chunk + static_cast<int64_t>(a.b.n_rows)) * heads);
    const int64_t run = 8 * static_cast<int64_t>(a.n_tiles), padded = (grid + run - 1) / run * run;
    if (padded > INT32_MAX)
        return tkv::set_error(TKV_EINVAL, "tkv_draft_verify: %lld workgroups are too many", static_cast<long long>(padded));
    draft_attn<D, R><<<dim3(static_cast<unsigned>(padded)), dim3(kThreads), 0, st>>>(a);
    return launched("tkv_draft_verify");
}

}  // namespace

int tkv::launch_draft_verify(const tkv_shape& s, const tkv_draft_batch& b, const DraftSplit& split, const void* q, const void* k,
                             const void* v, void* o, float* lse, void* ws, void* stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    Args a{};
    a.b = b;
    a.num_blocks = s.num_blocks, a.hq = s.hq, a.hkv = s.hkv, a.G = s.hq / s.hkv;
    a.chunk = split.chunk, a.n_chunks = split.n_chunks, a.n_tiles = split.n_tiles;
    a.sl2 = 1.4426950408889634f / sqrtf(static_cast<float>(s.d));
    a.q = static_cast<const uint16_t*>(q), a.k = static_cast<const uint16_t*>(k), a.v = static_cast<const uint16_t*>(v);
    a.o = static_cast<uint16_t*>(o), a.lse = lse;
    a.po = static_cast<float*>(ws);
    a.plse = a.po + static_cast<size_t>(a.n_chunks) * b.n_qtok * s.hq * s.d;
    int rc;
    if (s.d == 128)
        rc = split.waves == 4 ? launch<128, 4>(a, st) : launch<128, 2>(a, st);
    else
        rc = split.waves == 4 ? launch<64, 4>(a, st) : launch<64, 2>(a, st);
    if (rc != TKV_OK || a.n_chunks == 1) return rc;
    const auto merge = [&](auto kernel, int rows) -> int {  // rows: (token, head) rows a workgroup
        const int per_row = (b.max_q * s.hq + rows - 1) / rows;
        const int64_t grid = static_cast<int64_t>(per_row) * b.n_rows;
        if (grid > INT32_MAX) return tkv::set_error(TKV_EINVAL, "tkv_draft_verify: %d rows are too many", b.n_rows);
        kernel<<<dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, st>>>(a, per_row);
        return TKV_OK;
    };
    // Few rows share their chunks over four threads (896 rows of 32 chunks 4.8 us, 18 us with one a row); many rows fill
    // the chip by themselves (28,672 rows of up to 5 chunks 8.5 us, 16.7 us with four).
    constexpr int kParts = 4;
    const bool few = static_cast<int64_t>(b.n_qtok) * s.hq * (s.d / 4) * kParts <= 256 * 2048;
    if (s.d == 128)
        rc = few ? merge(draft_merge<128, kParts>, kThreads / (32 * kParts)) : merge(draft_merge<128, 1>, kThreads / 32);
    else
        rc = few ? merge(draft_merge<64, kParts>, kThreads / (16 * kParts)) : merge(draft_merge<64, 1>, kThreads / 16);
    if (rc != TKV_OK) return rc;
    return launched("tkv_draft_verify (merge)");
}
