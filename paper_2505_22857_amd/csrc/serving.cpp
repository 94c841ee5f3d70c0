// C ABI entry points of the serving operators that need no language model:
// verification, cache append and attention.  Argument checks and launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "trie.h"

namespace ngpu {
size_t verify_workspace(int64_t B, int K, int64_t V);
hipError_t launch_verify(const ngpu_verify_t &a, void *workspace, hipStream_t stream);
hipError_t launch_kv_append(const ngpu_kv_cache_t &c, const ngpu_kv_append_t &a, hipStream_t stream);
size_t attend_workspace(const ngpu_kv_cache_t &c, const ngpu_attend_t &a);
hipError_t launch_attend(const ngpu_kv_cache_t &c, const ngpu_attend_t &a, void *workspace, hipStream_t stream);
}  // namespace ngpu

namespace {

int refuse(const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return ngpu::set_error(NGPU_E_INVALID_ARG, buf);
}

int done(hipError_t e, const char *what) {
    if (e == hipSuccess) return ngpu::set_error(NGPU_OK, "");
    return ngpu::set_error(NGPU_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

int check_workspace(const void *p, size_t have, size_t need) {
    if (need == 0) return NGPU_OK;
    if (!p || have < need) return refuse("the workspace has %zu bytes, %zu are needed", p ? have : 0, need);
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return refuse("the workspace must be 16-byte aligned");
    return NGPU_OK;
}

// Rows times elements of a call: every index fits 62 bits.
constexpr int64_t kMostElements = int64_t(1) << 40;

int check_verify(const ngpu_verify_t *a) {
    if (!a) return refuse("null argument");
    if (a->B < 0 || a->B > NGPU_LM_MAX_SEQUENCES) return refuse("B = %lld outside [0, %d]", (long long)a->B,
                                                                NGPU_LM_MAX_SEQUENCES);
    if (a->K < 0 || a->K > NGPU_LM_MAX_DRAFT) return refuse("K = %d outside [0, %d]", a->K, NGPU_LM_MAX_DRAFT);
    if (a->V < 1 || a->V > INT32_MAX) return refuse("V = %lld outside [1, 2^31 - 1]", (long long)a->V);
    if (a->dtype != NGPU_F32 && a->dtype != NGPU_F16 && a->dtype != NGPU_BF16)
        return refuse("unknown type %d of the logits", a->dtype);
    const float t = a->temperature;
    if (t != 0.0f && !(std::isfinite(t) && t >= NGPU_LM_MIN_TEMPERATURE))
        return refuse("temperature must be 0 or finite and at least %g", NGPU_LM_MIN_TEMPERATURE);
    return NGPU_OK;
}

int check_cache(const ngpu_kv_cache_t *c) {
    if (!c) return refuse("null argument");
    if (c->dtype != NGPU_F16 && c->dtype != NGPU_BF16) return refuse("the cache holds half or bfloat16 values");
    if (c->dim < 1 || c->dim > NGPU_LM_MAX_HEAD_DIM)
        return refuse("dim = %d outside [1, %d]", c->dim, NGPU_LM_MAX_HEAD_DIM);
    if (c->heads < 1 || c->heads > 65536) return refuse("heads = %d outside [1, 65536]", c->heads);
    if (c->page_size < 1) return refuse("page_size = %d must be positive", c->page_size);
    if (c->num_pages < 0 || c->num_pages > INT32_MAX) return refuse("num_pages = %lld out of range",
                                                                    (long long)c->num_pages);
    if (c->k_stride_page < 0 || c->k_stride_token < 0 || c->k_stride_head < 0 || c->v_stride_page < 0 ||
        c->v_stride_token < 0 || c->v_stride_head < 0)
        return refuse("negative strides of the cache");
    if (c->num_pages > 0 && (!c->k || !c->v)) return refuse("null device pointer of the cache");
    return NGPU_OK;
}

int check_rows(int64_t S, int64_t T, int64_t heads, int64_t dim) {
    if (S < 0 || S > NGPU_LM_MAX_SEQUENCES) return refuse("S = %lld outside [0, %d]", (long long)S,
                                                          NGPU_LM_MAX_SEQUENCES);
    if (T < 0 || T > INT32_MAX) return refuse("T = %lld outside [0, 2^31 - 1]", (long long)T);
    if (heads < 0 || heads > 65536) return refuse("q_heads = %lld out of range", (long long)heads);
    if (S > 0 && T > 0 && S * T > kMostElements / (heads + 1) / dim) return refuse("the call is too large");
    return NGPU_OK;
}

int check_attend(const ngpu_kv_cache_t *c, const ngpu_attend_t *a) {
    if (const int rc = check_cache(c)) return rc;
    if (!a) return refuse("null argument");
    if (const int rc = check_rows(a->S, a->T, a->q_heads, c->dim)) return rc;
    if (a->q_heads < 1 || a->q_heads % c->heads != 0)
        return refuse("q_heads = %d is no multiple of the cache's %d heads", a->q_heads, c->heads);
    if (a->G < 0 || (a->G > 0 && a->S % a->G != 0))
        return refuse("%lld sequences do not divide into %lld groups", (long long)a->S, (long long)a->G);
    if (a->G > 0 && (a->prefix_width < 0 || a->prefix_width > INT32_MAX || a->prefix_stride < 0))
        return refuse("bad prefix tables");
    if (a->pages && (a->pages_width < 0 || a->pages_width > INT32_MAX || a->pages_stride < 0))
        return refuse("bad page tables");
    if (a->q_stride_seq < 0 || a->q_stride_token < 0 || a->q_stride_head < 0) return refuse("negative strides");
    if (!std::isfinite(a->scale)) return refuse("scale must be finite");
    return NGPU_OK;
}

}  // namespace

extern "C" {

size_t ngpu_lm_verify_workspace(int64_t B, int32_t K, int64_t V) {
    if (B <= 0 || B > NGPU_LM_MAX_SEQUENCES || K < 0 || K > NGPU_LM_MAX_DRAFT || V < 1 || V > INT32_MAX) return 0;
    return ngpu::verify_workspace(B, K, V);
}

int ngpu_lm_verify(const ngpu_verify_t *args, void *d_workspace, size_t workspace_bytes, void *hip_stream) {
    if (const int rc = check_verify(args)) return rc;
    const ngpu_verify_t &a = *args;
    if (a.B == 0) return done(hipSuccess, "");
    const bool sample = a.temperature != 0.0f;
    if (!a.logits || !a.out_tokens || !a.accepted || (a.K > 0 && !a.tokens) || (a.states && !a.draft_states) ||
        (sample && (!a.noise || (a.K > 0 && !a.uniforms))))
        return refuse("null device pointer");
    if (a.logits_stride_b < 0 || a.logits_stride_k < 0 || (sample && a.noise_stride_b < 0) ||
        (sample && a.logprobs && (a.logprobs_stride_b < 0 || a.logprobs_stride_k < 0)))
        return refuse("negative strides");
    if (const int rc = check_workspace(d_workspace, workspace_bytes, ngpu::verify_workspace(a.B, a.K, a.V))) return rc;
    return done(ngpu::launch_verify(a, d_workspace, static_cast<hipStream_t>(hip_stream)), "verify launch");
}

int ngpu_lm_kv_append(const ngpu_kv_cache_t *cache, const ngpu_kv_append_t *args, void *hip_stream) {
    if (const int rc = check_cache(cache)) return rc;
    if (!args) return refuse("null argument");
    ngpu_kv_append_t a = *args;
    if (!a.q) a.q_heads = 0;
    if (const int rc = check_rows(a.S, a.T, int64_t(a.q_heads) + 2 * cache->heads, cache->dim)) return rc;
    if (a.q && a.q_heads < 1) return refuse("q_heads = %d must be positive", a.q_heads);
    if (a.k_stride_seq < 0 || a.k_stride_token < 0 || a.k_stride_head < 0 || a.v_stride_seq < 0 ||
        a.v_stride_token < 0 || a.v_stride_head < 0 ||
        (a.q && (a.q_stride_seq < 0 || a.q_stride_token < 0 || a.q_stride_head < 0)))
        return refuse("negative strides");
    if (a.pages_width < 0 || a.pages_width > INT32_MAX || a.pages_stride < 0) return refuse("bad page tables");
    if (a.rotary < 0 || a.rotary > cache->dim || a.rotary % 2 != 0)
        return refuse("rotary = %d must be even and lie in [0, %d]", a.rotary, cache->dim);
    if (a.layout != NGPU_ROPE_HALF && a.layout != NGPU_ROPE_INTERLEAVED)
        return refuse("unknown rotation layout %d", a.layout);
    if (a.S == 0 || a.T == 0) return done(hipSuccess, "");
    if (!a.k || !a.v || !a.start || (!a.pages && a.pages_width > 0) || (a.q && !a.q_out) ||
        (a.rotary > 0 && a.positions_count > 0 && (!a.cos || !a.sin)))
        return refuse("null device pointer");
    if (a.q && a.q_out == a.q) return refuse("q_out must not overlap q");
    return done(ngpu::launch_kv_append(*cache, a, static_cast<hipStream_t>(hip_stream)), "append launch");
}

size_t ngpu_lm_attend_workspace(const ngpu_kv_cache_t *cache, const ngpu_attend_t *args) {
    if (check_attend(cache, args) != NGPU_OK) return 0;
    if (args->S == 0 || args->T == 0) return 0;
    return ngpu::attend_workspace(*cache, *args);
}

int ngpu_lm_attend(const ngpu_kv_cache_t *cache, const ngpu_attend_t *args, void *d_workspace,
                   size_t workspace_bytes, void *hip_stream) {
    if (const int rc = check_attend(cache, args)) return rc;
    const ngpu_attend_t &a = *args;
    if (a.S == 0 || a.T == 0) return done(hipSuccess, "");
    if (!a.q || !a.out || (a.G > 0 && (!a.prefix_lengths || (a.prefix_width > 0 && !a.prefix_pages))) ||
        (a.pages && !a.lengths))
        return refuse("null device pointer");
    if (const int rc = check_workspace(d_workspace, workspace_bytes, ngpu::attend_workspace(*cache, a))) return rc;
    return done(ngpu::launch_attend(*cache, a, d_workspace, static_cast<hipStream_t>(hip_stream)), "attend launch");
}

}  // extern "C"
