// Error reporting shared by every C entry point: a thread-local message behind tkv_last_error().
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

// ------------------------------------------------------------------ drafted trees: argument checks
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
