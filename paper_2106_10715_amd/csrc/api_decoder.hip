// C-ABI entry points of the operators around the expert layer in a decoder layer: argument checks.
#include <math.h>

#include "common.h"

using namespace moe;

namespace {

int check_norm(const moe_norm_cfg* c) {
    if (c == nullptr) return fail(MOE_ERR_INVALID_ARG, "cfg is NULL");
    if (c->dtype != MOE_F32 && c->dtype != MOE_BF16) return fail(MOE_ERR_INVALID_ARG, "dtype must be MOE_F32 or MOE_BF16");
    if (c->T < 0 || c->T >= 1 << 22) return fail(MOE_ERR_INVALID_ARG, "T must be in [0, 2^22) (got %d)", c->T);
    if (c->d < 8 || c->d > 32768 || c->d % 8 != 0) return fail(MOE_ERR_INVALID_ARG, "d must be a multiple of 8 in [8, 32768] (got %d)", c->d);
    if (c->q_group != 0 && c->q_group != 32 && c->q_group != 64 && c->q_group != 128)
        return fail(MOE_ERR_INVALID_ARG, "q_group must be 0, 32, 64 or 128 (got %d)", c->q_group);
    if (c->q_group != 0 && c->d % c->q_group != 0)
        return fail(MOE_ERR_INVALID_ARG, "q_group must divide d (got %d, d = %d)", c->q_group, c->d);
    if (!(c->eps > 0.f) || !isfinite(c->eps)) return fail(MOE_ERR_INVALID_ARG, "eps must be positive and finite");
    return MOE_OK;
}

int check_kv(const moe_kv_cfg* c) {
    if (c == nullptr) return fail(MOE_ERR_INVALID_ARG, "cfg is NULL");
    if (c->dtype != MOE_F32 && c->dtype != MOE_BF16) return fail(MOE_ERR_INVALID_ARG, "dtype must be MOE_F32 or MOE_BF16");
    if (c->cache_dtype != MOE_F32 && c->cache_dtype != MOE_BF16 && c->cache_dtype != MOE_E4M3)
        return fail(MOE_ERR_INVALID_ARG, "cache_dtype must be MOE_F32, MOE_BF16 or MOE_E4M3");
    if (c->cache_dtype == MOE_F32 && c->dtype != MOE_F32)
        return fail(MOE_ERR_UNSUPPORTED, "an fp32 cache needs fp32 activations");
    if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)) != 0)
        return fail(MOE_ERR_INVALID_ARG, "page_size must be a power of two in [16, 65536] (got %d)", c->page_size);
    if (c->pages < 1 || static_cast<long long>(c->pages) * c->page_size >= (1LL << 31))
        return fail(MOE_ERR_INVALID_ARG, "pages must be >= 1 and pages * page_size below 2^31 (got %d)", c->pages);
    if (c->heads < 1 || c->heads > 1024) return fail(MOE_ERR_INVALID_ARG, "heads must be in [1, 1024] (got %d)", c->heads);
    if (c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16 != 0)
        return fail(MOE_ERR_INVALID_ARG, "head_dim must be a multiple of 16 in [16, 256] (got %d)", c->head_dim);
    return MOE_OK;
}

int check_attn(const moe_kv_cfg* kv, const moe_attn_cfg* c) {
    if (int rc = check_kv(kv)) return rc;
    if (c == nullptr) return fail(MOE_ERR_INVALID_ARG, "attn is NULL");
    if (c->B < 0 || c->B > 4096) return fail(MOE_ERR_INVALID_ARG, "B must be in [0, 4096] (got %d)", c->B);
    if (c->q_heads < kv->heads || c->q_heads > 1024 || c->q_heads % kv->heads != 0)
        return fail(MOE_ERR_INVALID_ARG, "q_heads must be a multiple of heads, at most 1024 (got %d, heads = %d)", c->q_heads, kv->heads);
    if (c->table_pages < 1 || static_cast<long long>(c->table_pages) * kv->page_size > (1LL << 24))
        return fail(MOE_ERR_INVALID_ARG, "table_pages must be >= 1 and table_pages * page_size at most 2^24 (got %d)", c->table_pages);
    if (c->window < 0) return fail(MOE_ERR_INVALID_ARG, "window must be >= 0 (got %d)", c->window);
    if (!(c->scale >= 0.f) || !isfinite(c->scale)) return fail(MOE_ERR_INVALID_ARG, "scale must be finite and >= 0");
    return MOE_OK;
}

// The cache's arrays; the scales go with e4m3 and with nothing else.
int check_pages(const moe_kv_cfg& c, const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales) {
    REQUIRE(k_pages, "k_pages"); REQUIRE(v_pages, "v_pages");
    REQUIRE_ALIGNED(k_pages, "k_pages"); REQUIRE_ALIGNED(v_pages, "v_pages");
    if (c.cache_dtype == MOE_E4M3) {
        REQUIRE(k_scales, "k_scales"); REQUIRE(v_scales, "v_scales");
        REQUIRE_ALIGNED(k_scales, "k_scales"); REQUIRE_ALIGNED(v_scales, "v_scales");
    } else if (k_scales != nullptr || v_scales != nullptr) {
        return fail(MOE_ERR_INVALID_ARG, "scales are for an e4m3 cache");
    }
    return MOE_OK;
}

// Rows [n, heads * dim] of `stride` elements.
int check_rows(const void* p, int64_t stride, int64_t width, const char* name) {
    REQUIRE(p, name);
    REQUIRE_ALIGNED(p, name);
    if (stride < width || stride % 8 != 0 || stride >= (int64_t(1) << 31))
        return fail(MOE_ERR_INVALID_ARG, "the stride of %s must be a multiple of 8, at least %lld and below 2^31 (got %lld)", name,
                    static_cast<long long>(width), static_cast<long long>(stride));
    return MOE_OK;
}

int check_n(int32_t n) {
    if (n < 0) return fail(MOE_ERR_INVALID_ARG, "n must be >= 0 (got %d)", n);
    return MOE_OK;
}

}  // namespace

extern "C" {

int moe_add_norm(const moe_norm_cfg* cfg, const void* x, const void* residual, const void* weight, void* sum, void* y, void* q,
                 float* q_scale, void* stream) {
    if (int rc = check_norm(cfg)) return rc;
    REQUIRE(weight, "weight"); REQUIRE_ALIGNED(weight, "weight");
    if (cfg->T == 0) return MOE_OK;                                   // arrays without rows have no address
    if (y == nullptr && q == nullptr) return fail(MOE_ERR_INVALID_ARG, "y and q are both NULL");
    if ((q == nullptr) != (q_scale == nullptr)) return fail(MOE_ERR_INVALID_ARG, "q and q_scale go together");
    REQUIRE(x, "x"); REQUIRE_ALIGNED(x, "x");
    REQUIRE_ALIGNED(residual, "residual"); REQUIRE_ALIGNED(sum, "sum"); REQUIRE_ALIGNED(y, "y"); REQUIRE_ALIGNED(q, "q"); REQUIRE_ALIGNED(q_scale, "q_scale");
    return launch_add_norm(*cfg, x, residual, weight, sum, y, q, q_scale, static_cast<hipStream_t>(stream));
}

int moe_kv_write(const moe_kv_cfg* cfg, int32_t n, const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* slots,
                 void* k_pages, void* v_pages, float* k_scales, float* v_scales, void* stream) {
    if (int rc = check_kv(cfg)) return rc;
    if (int rc = check_n(n)) return rc;
    if (int rc = check_pages(*cfg, k_pages, v_pages, k_scales, v_scales)) return rc;
    if (n == 0) return MOE_OK;
    const int64_t width = static_cast<int64_t>(cfg->heads) * cfg->head_dim;
    if (int rc = check_rows(k, k_stride, width, "k")) return rc;
    if (int rc = check_rows(v, v_stride, width, "v")) return rc;
    REQUIRE(slots, "slots");
    return launch_kv_write(*cfg, n, k, k_stride, v, v_stride, slots, k_pages, v_pages, k_scales, v_scales, static_cast<hipStream_t>(stream));
}

int moe_kv_read(const moe_kv_cfg* cfg, int32_t n, const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales,
                const int32_t* slots, void* k, int64_t k_stride, void* v, int64_t v_stride, void* stream) {
    if (int rc = check_kv(cfg)) return rc;
    if (int rc = check_n(n)) return rc;
    if (int rc = check_pages(*cfg, k_pages, v_pages, k_scales, v_scales)) return rc;
    if (n == 0) return MOE_OK;
    const int64_t width = static_cast<int64_t>(cfg->heads) * cfg->head_dim;
    if (int rc = check_rows(k, k_stride, width, "k")) return rc;
    if (int rc = check_rows(v, v_stride, width, "v")) return rc;
    REQUIRE(slots, "slots");
    return launch_kv_read(*cfg, n, k_pages, v_pages, k_scales, v_scales, slots, k, k_stride, v, v_stride, static_cast<hipStream_t>(stream));
}

int moe_attn_workspace_bytes(const moe_kv_cfg* cfg, const moe_attn_cfg* attn, size_t* bytes) {
    if (int rc = check_attn(cfg, attn)) return rc;
    REQUIRE(bytes, "bytes");
    *bytes = attn_workspace_bytes(*cfg, *attn);
    return MOE_OK;
}

int moe_attn_decode(const moe_kv_cfg* cfg, const moe_attn_cfg* attn, const void* q, int64_t q_stride, const void* k_pages,
                    const void* v_pages, const float* k_scales, const float* v_scales, const int32_t* table, const int32_t* lens,
                    void* out, float* lse, void* ws, void* stream) {
    if (int rc = check_attn(cfg, attn)) return rc;
    if (int rc = check_pages(*cfg, k_pages, v_pages, k_scales, v_scales)) return rc;
    if (attn->B == 0) return MOE_OK;
    if (int rc = check_rows(q, q_stride, static_cast<int64_t>(attn->q_heads) * cfg->head_dim, "q")) return rc;
    REQUIRE(table, "table"); REQUIRE(lens, "lens"); REQUIRE(out, "out"); REQUIRE(ws, "ws");
    REQUIRE_ALIGNED(out, "out");
    if ((reinterpret_cast<uintptr_t>(ws) & 255) != 0) return fail(MOE_ERR_WORKSPACE, "ws must be 256-byte aligned");
    return launch_attn_decode(*cfg, *attn, q, q_stride, k_pages, v_pages, k_scales, v_scales, table, lens, out, lse, ws,
                              static_cast<hipStream_t>(stream));
}

}  // extern "C"
