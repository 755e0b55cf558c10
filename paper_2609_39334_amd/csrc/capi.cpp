// Error reporting shared by every C entry point (a thread-local message behind tkv_last_error()), and the host halves of
// the entry points that take device data alone: their checks of arguments, and how a drafted batch is cut.
#include <algorithm>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <string>

#include "internal.h"

namespace {
thread_local std::string g_error;
}

namespace tkv {

int set_error(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    g_error = buf;
    return code;
}

void clear_error() { g_error.clear(); }

}  // namespace tkv

TKV_EXPORT const char* tkv_last_error(void) { return g_error.c_str(); }

// ------------------------------------------------------------------ norms with the append, drafted trees, truncated draws
namespace {

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// The pool's shape, as the device entry points below take it; an error is recorded.
int check_pool(const char* fn, const tkv_shape* s) {
    if (!s) return tkv::set_error(TKV_EINVAL, "%s: shape is NULL", fn);
    if (s->block_size != tkv::kBlock) return tkv::set_error(TKV_EINVAL, "%s: block_size must be 16 (got %d)", fn, s->block_size);
    if (s->d != 64 && s->d != 128) return tkv::set_error(TKV_EINVAL, "%s: head_dim must be 64 or 128 (got %d)", fn, s->d);
    if (s->hq < 1 || s->hkv < 1 || s->num_blocks < 1)
        return tkv::set_error(TKV_EINVAL, "%s: hq, hkv and num_blocks must be >= 1", fn);
    if (static_cast<int64_t>(s->num_blocks) * s->block_size > INT32_MAX)
        return tkv::set_error(TKV_EINVAL, "%s: %d blocks exceed the int32 slot range", fn, s->num_blocks);
    return TKV_OK;
}

}  // namespace

TKV_EXPORT int tkv_norm_rope_append(const tkv_shape* shape, int32_t n_tok, const void* qkv, int64_t qkv_stride,
                                    const float* q_weight, const float* k_weight, float eps, const float* cosv,
                                    const float* sinv, int32_t rot, const int32_t* d_dst, void* q, void* k, void* v,
                                    void* stream) {
    const char* fn = "tkv_norm_rope_append";
    tkv::clear_error();
    if (const int rc = check_pool(fn, shape)) return rc;
    const int64_t width = (static_cast<int64_t>(shape->hq) + 2 * static_cast<int64_t>(shape->hkv)) * shape->d;
    if (rot < 0 || rot > shape->d || rot % 16 != 0)
        return tkv::set_error(TKV_EINVAL, "%s: rot must be a multiple of 16 up to head_dim (got %d)", fn, rot);
    if (qkv_stride < width || qkv_stride % 8 != 0)
        return tkv::set_error(TKV_EINVAL, "%s: qkv_stride must be a multiple of 8, at least %lld (got %lld)", fn,
                              static_cast<long long>(width), static_cast<long long>(qkv_stride));
    if (n_tok < 0) return tkv::set_error(TKV_EINVAL, "%s: n_tok = %d < 0", fn, n_tok);
    if (n_tok == 0) return TKV_OK;
    if (!qkv || !q_weight || !k_weight || !d_dst || !q || !k || !v || (rot > 0 && (!cosv || !sinv)))
        return tkv::set_error(TKV_EINVAL, "%s: NULL pointer", fn);
    for (const void* p : {qkv, static_cast<const void*>(q_weight), static_cast<const void*>(k_weight),
                          static_cast<const void*>(cosv), static_cast<const void*>(sinv), static_cast<const void*>(q),
                          static_cast<const void*>(k), static_cast<const void*>(v)})
        if (!aligned16(p)) return tkv::set_error(TKV_EINVAL, "%s: tensors must be 16-byte aligned", fn);
    if (!tkv::launch_norm_rope_append) return tkv::set_error(TKV_EHIP, "%s: host-only build, no device", fn);
    return tkv::launch_norm_rope_append(*shape, n_tok, qkv, qkv_stride, q_weight, k_weight, eps, cosv, sinv, rot, d_dst, q, k,
                                        v, stream);
}

TKV_EXPORT int tkv_draft_mask(int32_t n, const int32_t* parent, int32_t words, uint64_t* mask_out, int32_t* depth_out) {
    tkv::clear_error();
    if (n < 0 || (n > 0 && !parent)) return tkv::set_error(TKV_EINVAL, "tkv_draft_mask: n %d, parent %p", n, static_cast<const void*>(parent));
    if (mask_out && words < (static_cast<int64_t>(n) + 63) / 64)
        return tkv::set_error(TKV_EINVAL, "tkv_draft_mask: %d words do not hold %d tokens", words, n);
    for (int32_t i = 0; i < n; ++i)
        if (parent[i] < -1 || parent[i] >= i)
            return tkv::set_error(TKV_EINVAL, "tkv_draft_mask: parent[%d] = %d is not an earlier token or -1", i, parent[i]);
    for (int32_t i = 0; i < n; ++i) {
        const int32_t p = parent[i];
        if (mask_out) {
            uint64_t* row = mask_out + static_cast<size_t>(i) * words;
            for (int32_t w = 0; w < words; ++w) row[w] = p < 0 ? 0 : mask_out[static_cast<size_t>(p) * words + w];
            row[i / 64] |= uint64_t{1} << (i % 64);
        }
        if (depth_out) depth_out[i] = p < 0 ? 0 : depth_out[p] + 1;
    }
    return TKV_OK;
}

namespace {

constexpr int32_t kMaxDraft = 1024;  // query tokens of a row
constexpr int32_t kMinDraftChunk = 16, kLongDraftChunk = 192, kMaxDraftChunk = 256, kShortDraft = 32;  // blocks
constexpr int64_t kFewDraftRows = 4096;

int check_draft(const char* fn, const tkv_shape* s, const tkv_draft_batch* b) {
    if (const int rc = check_pool(fn, s)) return rc;
    if (s->hq % s->hkv != 0) return tkv::set_error(TKV_EINVAL, "%s: hq (%d) must be a multiple of hkv (%d)", fn, s->hq, s->hkv);
    if (s->hq / s->hkv > tkv::kTileRows || s->hq > 256)
        return tkv::set_error(TKV_EINVAL, "%s: hq = %d (up to 256), hq/hkv = %d (up to %d)", fn, s->hq, s->hq / s->hkv, tkv::kTileRows);
    if (!b) return tkv::set_error(TKV_EINVAL, "%s: batch is NULL", fn);
    if (b->n_rows < 0 || b->n_qtok < 0 || b->n_kv_blocks < 0)
        return tkv::set_error(TKV_EINVAL, "%s: n_rows %d, n_qtok %d, n_kv_blocks %d", fn, b->n_rows, b->n_qtok, b->n_kv_blocks);
    if (b->max_q < 1 || b->max_q > kMaxDraft) return tkv::set_error(TKV_EINVAL, "%s: max_q = %d is not in [1, %d]", fn, b->max_q, kMaxDraft);
    if (b->max_blocks < 1) return tkv::set_error(TKV_EINVAL, "%s: max_blocks = %d < 1", fn, b->max_blocks);
    if (b->mask_words < (b->max_q + 63) / 64)
        return tkv::set_error(TKV_EINVAL, "%s: %d mask words do not hold %d tokens", fn, b->mask_words, b->max_q);
    return TKV_OK;
}

// Tiles of 64 query rows, whose two pairs of waves share the keys, where the batch has no wider row or few rows in all
// (little between them there: one row of 32 tokens, 28/4/128 heads, 30,000 keys 36 us against 37 with tiles of 128; 64
// single tokens of 12/2/128 heads under 300 to 6,144 keys 39 against 40), else 128 (32 rows of 4 to 32 tokens, 28/4/128:
// 64 against 70).
// Chunks as long as they can be with a unit for every slot of the chip (two workgroups a CU for heads of 128, three
// for 64): a unit costs about 7 us beside its stages, and one past the slots waits for a whole round (those 32 rows:
// 484 units of up to 104 blocks 66 us, 528 of up to 93 78 us, 728 of 64 83 us).  Chunks that would pass 192 blocks
// are cut for two rounds, or more (8 rows of 64 to 150 tokens, 32/8/128, 2,000 to 12,000 keys: 178 us with 150
// blocks, 211 with 240).  A row's chunks are whole in number, of near-equal length, so tables make more units than their
// blocks fill: `uneven`, too much for long rows (those 8 rows: 856 units of 128 to 164 blocks on the 1,024 slots of two
// rounds).
// Where the longest table has 32 blocks the merge costs more than a split saves (64 rows under 20 to 300 keys 13.5 us,
// 20 us in chunks of 16).
tkv::DraftSplit draft_split(const tkv_shape& s, const tkv_draft_batch& b) {
    tkv::DraftSplit x{};
    const int64_t G = s.hq / s.hkv, rows = b.max_q * G;
    x.waves = rows <= 64 || static_cast<int64_t>(b.n_qtok) * s.hq <= kFewDraftRows ? 2 : 4;
    const int64_t tile_rows = 32 * x.waves;
    x.n_tiles = static_cast<int32_t>((rows + tile_rows - 1) / tile_rows);
    const double n_rows = b.n_rows > 0 ? b.n_rows : 1;
    const double tiles = std::min<double>(x.n_tiles, std::max(1., b.n_qtok / n_rows * static_cast<double>(G) / static_cast<double>(tile_rows) + .5));
    const double work = b.n_kv_blocks * tiles * s.hkv, uneven = .8 * n_rows * s.hkv * tiles, slots = s.d == 128 ? 512 : 768;
    double chunk = kMaxDraftChunk;
    for (int k = 1; k <= 64; ++k) {
        const double units = slots * k - uneven;
        if (units > 0 && work / units <= kLongDraftChunk) {
            chunk = work / units;
            break;
        }
    }
    x.chunk = static_cast<int32_t>(std::min<double>(kMaxDraftChunk, std::max<double>(kMinDraftChunk, chunk)));
    x.chunk = (x.chunk + 3) & ~3;
    const int64_t longest = std::min(b.max_blocks, b.n_kv_blocks);
    if (longest <= kShortDraft) x.chunk = kMaxDraftChunk;
    x.n_chunks = static_cast<int32_t>(longest > x.chunk ? (longest + x.chunk - 1) / x.chunk : 1);
    if (x.n_chunks > 1)
        x.bytes = static_cast<size_t>(x.n_chunks) * static_cast<size_t>(b.n_qtok) * static_cast<size_t>(s.hq) *
                  (static_cast<size_t>(s.d) + 1) * sizeof(float);
    return x;
}

}  // namespace

TKV_EXPORT int tkv_draft_workspace_bytes(const tkv_shape* shape, const tkv_draft_batch* batch, size_t* bytes_out) {
    const char* fn = "tkv_draft_workspace_bytes";
    tkv::clear_error();
    if (!bytes_out) return tkv::set_error(TKV_EINVAL, "%s: bytes_out is NULL", fn);
    if (const int rc = check_draft(fn, shape, batch)) return rc;
    *bytes_out = draft_split(*shape, *batch).bytes;
    return TKV_OK;
}

TKV_EXPORT int tkv_draft_verify(const tkv_shape* shape, const tkv_draft_batch* batch, const void* q, const void* k,
                                const void* v, void* o, float* lse, void* d_workspace, size_t bytes, void* stream) {
    const char* fn = "tkv_draft_verify";
    tkv::clear_error();
    if (const int rc = check_draft(fn, shape, batch)) return rc;
    const tkv_draft_batch& b = *batch;
    if (b.n_rows == 0 || b.n_qtok == 0) return TKV_OK;
    if (!b.q_indptr || !b.kv_indptr || !b.block_len || !b.mask || (b.n_kv_blocks > 0 && !b.kv_blocks) || !q || !k || !v || !o)
        return tkv::set_error(TKV_EINVAL, "%s: NULL pointer", fn);
    for (const void* p : {q, k, v, static_cast<const void*>(o), static_cast<const void*>(d_workspace)})
        if (!aligned16(p)) return tkv::set_error(TKV_EINVAL, "%s: tensors must be 16-byte aligned", fn);
    const tkv::DraftSplit split = draft_split(*shape, b);
    if (split.bytes > 0 && (!d_workspace || bytes < split.bytes))
        return tkv::set_error(TKV_EINVAL, "%s: workspace of %zu bytes < %zu needed", fn, d_workspace ? bytes : 0, split.bytes);
    if (!tkv::launch_draft_verify) return tkv::set_error(TKV_EHIP, "%s: host-only build, no device", fn);
    return tkv::launch_draft_verify(*shape, b, split, q, k, v, o, lse, d_workspace, stream);
}

namespace {
constexpr int32_t kMaxFilterVocab = 1 << 21, kMaxFilterPotential = 1024;
}

TKV_EXPORT size_t tkv_filter_sample_workspace_bytes(int32_t n_rows, int32_t vocab) {
    tkv::clear_error();
    if (n_rows <= 0 || vocab <= 0) return 0;
    return tkv::filter_layout(n_rows, vocab).bytes;
}

TKV_EXPORT int tkv_filter_sample(int32_t n_rows, int32_t vocab, int32_t logit_type, const void* d_logits, int64_t stride,
                                 const float* d_temperature, const int32_t* d_top_k, const float* d_top_p,
                                 const float* d_min_p, int32_t max_potential, const float* d_uniform,
                                 const int32_t* d_draw_off, int32_t n_draws, int32_t* d_token, int32_t* d_count,
                                 int32_t* d_n_groups, void* d_workspace, size_t bytes, void* stream) {
    const char* fn = "tkv_filter_sample";
    tkv::clear_error();
    if (n_rows < 0 || vocab < 1) return tkv::set_error(TKV_EINVAL, "%s: n_rows %d, vocab %d", fn, n_rows, vocab);
    if (vocab > kMaxFilterVocab) return tkv::set_error(TKV_EINVAL, "%s: vocabulary %d exceeds %d", fn, vocab, kMaxFilterVocab);
    if (logit_type != TKV_LOGITS_F32 && logit_type != TKV_LOGITS_BF16)
        return tkv::set_error(TKV_EINVAL, "%s: logit_type %d", fn, logit_type);
    if (stride < vocab) return tkv::set_error(TKV_EINVAL, "%s: stride %lld < vocab %d", fn, static_cast<long long>(stride), vocab);
    if (max_potential < 0 || max_potential > kMaxFilterPotential)
        return tkv::set_error(TKV_EINVAL, "%s: potential up to %d per row (got %d)", fn, kMaxFilterPotential, max_potential);
    if (n_draws < 0) return tkv::set_error(TKV_EINVAL, "%s: n_draws = %d < 0", fn, n_draws);
    if (n_rows == 0) return TKV_OK;
    if (!d_logits || !d_temperature || !d_draw_off || !d_n_groups || (n_draws > 0 && (!d_uniform || !d_token || !d_count)))
        return tkv::set_error(TKV_EINVAL, "%s: NULL pointer", fn);
    const size_t need = tkv_filter_sample_workspace_bytes(n_rows, vocab);
    if (need > 0 && (!d_workspace || bytes < need))
        return tkv::set_error(TKV_EINVAL, "%s: workspace of %zu bytes < %zu needed", fn, d_workspace ? bytes : 0, need);
    if (!aligned16(d_workspace)) return tkv::set_error(TKV_EINVAL, "%s: workspace not 16-byte aligned", fn);
    if (!tkv::launch_filter_sample) return tkv::set_error(TKV_EHIP, "%s: host-only build, no device", fn);
    tkv::FilterCall f{};
    f.n_rows = n_rows, f.vocab = vocab, f.logit_type = logit_type, f.n_draws = n_draws;
    f.logits = d_logits, f.stride = stride;
    f.temperature = d_temperature, f.top_k = d_top_k, f.top_p = d_top_p, f.min_p = d_min_p;
    f.uniform = d_uniform, f.draw_off = d_draw_off;
    f.token = d_token, f.count = d_count, f.n_groups = d_n_groups, f.workspace = d_workspace;
    return tkv::launch_filter_sample(f, stream);
}
