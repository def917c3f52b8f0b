// Entry points of the paged cache and of sampling: argument checks, then the launches on the
// caller's stream.  Host side only.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "kernels.h"
#include "prepack.h"
#include "status.h"

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxHeadRows = 1 << 22;   // sequences times query heads: a launch holds fewer than 2^32 threads
constexpr int32_t kMaxVocab = (1 << 20) - 1;   // sums of weights of up to 2^44 fit 64 bits

bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; }

pp_status finish(const char* what) {
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return pp::fail(PP_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(err));
    return PP_OK;
}

// Sizes of the config and the cache.
pp_status check_sizes(const pp_config* cfg, const pp_paged_cache* c) {
    if (pp_status st = pp::validate_config(cfg)) return st;
    if (!c) return pp::fail(PP_ERR_INVALID_ARG, "cache is NULL");
    if (c->kv_type < PP_KV_F32 || c->kv_type > PP_KV_I8)
        return pp::fail(PP_ERR_INVALID_ARG, "unknown kv_type %d", c->kv_type);
    if (c->k < 0 || c->max_pages < 0 || c->n_pages <= 0 || c->page_size <= 0)
        return pp::fail(PP_ERR_INVALID_ARG, "k %d, max_pages %d, n_pages %d, page_size %d", c->k, c->max_pages,
                        c->n_pages, c->page_size);
    if (c->kv_type != PP_KV_I8 && (c->kv_type == PP_KV_F32) != (cfg->dtype == PP_F32))
        return pp::fail(PP_ERR_UNSUPPORTED, "kv_type %d with dtype %d: pages hold the config's dtype or 8-bit codes",
                        c->kv_type, cfg->dtype);
    if (c->page_size & (c->page_size - 1))
        return pp::fail(PP_ERR_UNSUPPORTED, "page_size %d is not a power of two", c->page_size);
    if (int64_t(c->n_pages) * c->page_size > INT32_MAX)
        return pp::fail(PP_ERR_UNSUPPORTED, "%d pages of %d rows are more than 2^31 - 1 rows", c->n_pages, c->page_size);
    if (int64_t(c->k) * cfg->n_heads > kMaxHeadRows)
        return pp::fail(PP_ERR_UNSUPPORTED, "k * n_heads above %lld", (long long)kMaxHeadRows);
    return PP_OK;
}

// Its buffers.
pp_status check_buffers(const pp_paged_cache* c) {
    if ((int64_t(c->k) * c->max_pages > 0 && !c->page_table) || !c->k_pages || !c->v_pages ||
        (c->kv_type == PP_KV_I8 && (!c->k_scale || !c->v_scale)))
        return pp::fail(PP_ERR_INVALID_ARG, "a buffer of the cache is NULL");
    if (misaligned(c->k_pages) || misaligned(c->v_pages))
        return pp::fail(PP_ERR_UNSUPPORTED, "pages must be 16-byte aligned");
    return PP_OK;
}

ppk::PagedCache view(const pp_config* cfg, const pp_paged_cache* c) {
    return {c->kv_type, c->k, __builtin_ctz(c->page_size), c->max_pages, c->n_pages, c->page_table, c->k_pages,
            c->v_pages, c->k_scale, c->v_scale, cfg->n_heads, cfg->n_kv_heads, cfg->head_dim};
}

pp_status check_workspace(const void* ws, size_t bytes, size_t need) {
    if (!need) return PP_OK;
    if (!ws) return pp::fail(PP_ERR_INVALID_ARG, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(ws) % kAlign)
        return pp::fail(PP_ERR_INVALID_ARG, "workspace is not %zu-byte aligned", kAlign);
    if (bytes < need) return pp::fail(PP_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes < %zu needed", bytes, need);
    return PP_OK;
}

// What pp_paged_write and pp_paged_read share; *done: there is nothing to do.
pp_status check_rows(const pp_config* cfg, const pp_paged_cache* c, const int32_t* seq, const int32_t* pos, int32_t rows,
                     const void* k, int64_t ldk, const void* v, int64_t ldv, bool* done) {
    *done = false;
    if (pp_status st = check_sizes(cfg, c)) return st;
    const int64_t kvw = int64_t(cfg->n_kv_heads) * cfg->head_dim;
    if (rows < 0) return pp::fail(PP_ERR_INVALID_ARG, "rows %d", rows);
    if (ldk < kvw || ldv < kvw)
        return pp::fail(PP_ERR_INVALID_ARG, "row strides %lld, %lld below Hkv D", (long long)ldk, (long long)ldv);
    if (ldk % 8 || ldv % 8)
        return pp::fail(PP_ERR_UNSUPPORTED, "row strides %lld, %lld must be multiples of 8", (long long)ldk, (long long)ldv);
    *done = rows == 0 || c->k == 0;
    if (*done) return PP_OK;
    if (!seq || !pos || !k || !v) return pp::fail(PP_ERR_INVALID_ARG, "NULL buffer");
    if (misaligned(k) || misaligned(v)) return pp::fail(PP_ERR_UNSUPPORTED, "keys and values must be 16-byte aligned");
    return check_buffers(c);
}

}  // namespace

extern "C" pp_status pp_paged_write(const pp_config* cfg, const pp_paged_cache* cache, const int32_t* seq,
                                    const int32_t* pos, int32_t rows, const void* keys, int64_t ldk,
                                    const void* values, int64_t ldv, void* stream) {
    pp::clear_error();
    bool done;
    if (pp_status st = check_rows(cfg, cache, seq, pos, rows, keys, ldk, values, ldv, &done)) return st;
    if (done) return PP_OK;
    (void)hipGetLastError();
    ppk::paged_write(cfg->dtype, view(cfg, cache), seq, pos, rows, keys, ldk, values, ldv, static_cast<hipStream_t>(stream));
    return finish("paged_write");
}

extern "C" pp_status pp_paged_read(const pp_config* cfg, const pp_paged_cache* cache, const int32_t* seq,
                                   const int32_t* pos, int32_t rows, void* keys, int64_t ldk, void* values, int64_t ldv,
                                   void* stream) {
    pp::clear_error();
    bool done;
    if (pp_status st = check_rows(cfg, cache, seq, pos, rows, keys, ldk, values, ldv, &done)) return st;
    if (done) return PP_OK;
    (void)hipGetLastError();
    ppk::paged_read(cfg->dtype, view(cfg, cache), seq, pos, rows, keys, ldk, values, ldv, static_cast<hipStream_t>(stream));
    return finish("paged_read");
}

extern "C" pp_status pp_paged_append(const pp_config* cfg, const pp_paged_cache* cache, const int32_t* lens,
                                     const void* qkv, int64_t ldqkv, void* q_out, int64_t ldq, void* stream) {
    pp::clear_error();
    if (pp_status st = check_sizes(cfg, cache)) return st;
    const int64_t D = cfg->head_dim;
    if (ldqkv < (cfg->n_heads + 2 * int64_t(cfg->n_kv_heads)) * D || ldq < cfg->n_heads * D)
        return pp::fail(PP_ERR_INVALID_ARG, "ldqkv %lld or ldq %lld below its row", (long long)ldqkv, (long long)ldq);
    if (ldqkv % 8 || ldq % 8)
        return pp::fail(PP_ERR_UNSUPPORTED, "ldqkv %lld and ldq %lld must be multiples of 8", (long long)ldqkv, (long long)ldq);
    if (cache->k == 0) return PP_OK;
    if (!lens || !qkv || !q_out) return pp::fail(PP_ERR_INVALID_ARG, "NULL buffer");
    if (misaligned(qkv) || misaligned(q_out)) return pp::fail(PP_ERR_UNSUPPORTED, "qkv and q_out must be 16-byte aligned");
    if (qkv == q_out && ldqkv != ldq) return pp::fail(PP_ERR_INVALID_ARG, "q_out is qkv, with another row stride");
    if (pp_status st = check_buffers(cache)) return st;
    (void)hipGetLastError();
    ppk::paged_append(cfg->dtype, view(cfg, cache), lens, qkv, ldqkv, q_out, ldq, cfg->rope_theta,
                      static_cast<hipStream_t>(stream));
    return finish("paged_append");
}

extern "C" pp_status pp_paged_attention_workspace_size(const pp_config* cfg, const pp_paged_cache* cache, size_t* bytes) {
    pp::clear_error();
    if (pp_status st = check_sizes(cfg, cache)) return st;
    if (!bytes) return pp::fail(PP_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = ppk::paged_attention_workspace(cache->k, cfg->n_heads, cfg->n_kv_heads, cfg->head_dim);
    return PP_OK;
}

extern "C" pp_status pp_paged_attention(const pp_config* cfg, const pp_paged_cache* cache, const int32_t* lens,
                                        const void* q, int64_t ldq, void* out, void* workspace, size_t workspace_bytes,
                                        void* stream) {
    pp::clear_error();
    if (pp_status st = check_sizes(cfg, cache)) return st;
    if (ldq < int64_t(cfg->n_heads) * cfg->head_dim) return pp::fail(PP_ERR_INVALID_ARG, "ldq %lld < H*D", (long long)ldq);
    if (ldq % 8) return pp::fail(PP_ERR_UNSUPPORTED, "ldq %lld must be a multiple of 8", (long long)ldq);
    if (cache->k == 0) return PP_OK;
    if (!lens || !q || !out) return pp::fail(PP_ERR_INVALID_ARG, "NULL buffer");
    if (misaligned(q) || misaligned(out)) return pp::fail(PP_ERR_UNSUPPORTED, "q and out must be 16-byte aligned");
    if (pp_status st = check_buffers(cache)) return st;
    const size_t need = ppk::paged_attention_workspace(cache->k, cfg->n_heads, cfg->n_kv_heads, cfg->head_dim);
    if (pp_status st = check_workspace(workspace, workspace_bytes, need)) return st;
    (void)hipGetLastError();
    ppk::paged_attention(cfg->dtype, view(cfg, cache), lens, q, ldq, out, workspace, static_cast<hipStream_t>(stream));
    return finish("paged_attention");
}

namespace {
pp_status check_vocab(int32_t k, int32_t vocab) {
    if (k < 0 || vocab <= 0) return pp::fail(PP_ERR_INVALID_ARG, "k %d, vocab %d", k, vocab);
    if (vocab > kMaxVocab) return pp::fail(PP_ERR_UNSUPPORTED, "vocab %d above %d", vocab, kMaxVocab);
    if (k > kMaxHeadRows / 4) return pp::fail(PP_ERR_UNSUPPORTED, "k %d above %lld", k, (long long)kMaxHeadRows / 4);
    return PP_OK;
}
}  // namespace

extern "C" pp_status pp_sample_workspace_size(int32_t k, int32_t vocab, size_t* bytes) {
    pp::clear_error();
    if (pp_status st = check_vocab(k, vocab)) return st;
    if (!bytes) return pp::fail(PP_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = ppk::sample_workspace(k, vocab);
    return PP_OK;
}

extern "C" pp_status pp_sample(const float* logits, int64_t ldl, int32_t k, int32_t vocab, const float* temperature,
                               const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                               void* workspace, size_t workspace_bytes, int32_t* tokens, float* prob, void* stream) {
    pp::clear_error();
    if (pp_status st = check_vocab(k, vocab)) return st;
    if (ldl < vocab) return pp::fail(PP_ERR_INVALID_ARG, "ldl %lld < vocab", (long long)ldl);
    if (k == 0) return PP_OK;
    if (!logits || !u || !tokens) return pp::fail(PP_ERR_INVALID_ARG, "NULL buffer");
    if (pp_status st = check_workspace(workspace, workspace_bytes, ppk::sample_workspace(k, vocab))) return st;
    (void)hipGetLastError();
    ppk::sample(ppk::Sample{logits, ldl, k, vocab, temperature, top_k, top_p, min_p, u, tokens, prob, workspace},
                static_cast<hipStream_t>(stream));
    return finish("sample");
}
